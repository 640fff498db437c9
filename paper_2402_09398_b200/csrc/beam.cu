// The selection of beam search: of the candidates (beam, token) of a group the `keep` largest
//
//   v(b, t) = score_b + l(b, t) - log sum_u exp l(b, u),     ties to the lowest (b, t)
//
// Bound by memory: every logit of a live beam is read once (2 or 4 bytes; an exponential, a sum and two comparisons each).
//   - A row of logits is cut over several CTAs.  Each takes its stretch in one pass: sum of exponentials relative to a
//     reference (the largest logit of its first tile; moved only where a later one lies more than 2^57 above), and its
//     `keep` largest logits.  Those pass a bar: the keep-th largest of the maxima of 64 (256) groups of threads over the
//     first tile, which at least `keep` elements reach and, of n elements like those of the tile, about keep n / tile.
//     They go to a list in shared memory, from which the largest are taken by counting for each how many are larger.
//   - The CTA of a group that arrives last joins: the rows' sums, then the candidates of all beams the same way.
// Within a beam the order is that of the logits, which is exact.  Between beams it hangs on the sums.  Their fp32
// arithmetic is off by at most 2 * 2^-22 (exponentials) + 17 * 2^-23.2 (their arguments, whose mean distance from the largest
// is at most log2 of the number of tokens) + 8 * 2^-24 (a thread's sum over a tile; the rest is in 64 bits), 2.8e-6 in all;
// so where two neighbours in the order are of different beams and closer than kClose, the sums of these beams are computed
// again in 64 bits and the candidates joined once more.  (Chances are some 1e-4 per kept candidate.)
#include <float.h>

#include "less_internal.cuh"
#include "pages_attn.cuh"

namespace less {

constexpr int BM_THREADS = 256, BM_UNROLL = 4;            // 16-byte pieces of a thread on their way
constexpr int BM_TILE = BM_THREADS * BM_UNROLL;           // 16-byte pieces of a tile
constexpr int BM_LIST = 2048;                             // candidates that a list holds
constexpr int BM_MOST_BEAMS = 64, BM_MOST_KEEP = 128;
constexpr int BM_JOINED = 8192;                           // candidates of a group that are joined, about
constexpr int BM_DIRECT = 512;                            // as many are compared with one another at once
constexpr float kRefFar = 40.f;                           // a logit that far above the reference moves it
constexpr double kClose = 0x1p-17;                        // more than the errors of two sums

struct BmArgs {
  const void* logits;
  int64_t stride;                                         // elements from row to row
  const float* scores;
  const uint8_t* ended;                                   // or null
  int groups, beams, vocab, keep, end_token, splits, per; // per: 16-byte pieces of a CTA
  float* out_scores;
  int32_t* out_tokens;
  int32_t* out_parents;
  uint8_t* out_ended;
  int32_t* counters;                                      // [groups] zero between calls
  float2* sums;                                           // [rows][splits] (reference, sum)
  unsigned long long* keys;                               // [rows][splits][keep]
};

template <typename T>
struct BmType;
template <>
struct BmType<float> {
  static constexpr int N = 4;                             // elements of 16 bytes
  static constexpr float most = FLT_MAX;
  static __device__ __forceinline__ void unpack(uint4 w, float* f) {    // NaN counts as -inf
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = fmaxf(__uint_as_float(u[i]), -INFINITY);
  }
  static __device__ __forceinline__ float load(const void* p) { return fmaxf(__ldcg((const float*)p), -INFINITY); }
};
template <>
struct BmType<__half> {
  static constexpr int N = 8;
  static constexpr float most = 65504.f;
  static __device__ __forceinline__ void unpack(uint4 w, float* f) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    const __half2 low = __half2half2(__ushort_as_half(0xfc00));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = __half22float2(__hmax2(*reinterpret_cast<const __half2*>(&u[i]), low));
      f[2 * i] = x.x;
      f[2 * i + 1] = x.y;
    }
  }
  static __device__ __forceinline__ float load(const void* p) {
    return fmaxf(__half2float(__ushort_as_half(__ldcg((const unsigned short*)p))), -INFINITY);
  }
};
template <>
struct BmType<__nv_bfloat16> {
  static constexpr int N = 8;
  static constexpr float most = 3.38953138925153547590470800371487866880e+38f;
  static __device__ __forceinline__ void unpack(uint4 w, float* f) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    const __nv_bfloat162 low = __bfloat162bfloat162(__ushort_as_bfloat16(0xff80));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 c = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&u[i]), low);
      const uint32_t x = *reinterpret_cast<const uint32_t*>(&c);
      f[2 * i] = __uint_as_float(x << 16);
      f[2 * i + 1] = __uint_as_float(x & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ float load(const void* p) {
    return fmaxf(__uint_as_float((uint32_t)__ldcg((const unsigned short*)p) << 16), -INFINITY);
  }
};

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
  unsigned long long at;                                  // beam << 32 | token, ~0 = none
};
constexpr long long kNoCand = (long long)0x8000000000000000ull;
__device__ __forceinline__ long long bm_order(double v) {
  const long long b = __double_as_longlong(v + 0.0);      // the two zeros are equal
  return b ^ (b >> 63 & 0x7fffffffffffffffll);
}
__device__ __forceinline__ double bm_value(long long o) { return __longlong_as_double(o ^ (o >> 63 & 0x7fffffffffffffffll)); }
__device__ __forceinline__ bool bm_before(const BmCand& a, const BmCand& b) { return a.v > b.v || (a.v == b.v && a.at < b.at); }

struct BmShared {
  union {
    unsigned long long list[BM_LIST];
    struct {
      BmCand cand[BM_LIST / 2];
      double score[BM_MOST_BEAMS], lse[BM_MOST_BEAMS];    // -inf = no candidates
    } j;
  };
  union {
    float best[BM_THREADS];
    BmCand most[BM_THREADS];
    unsigned long long high[BM_THREADS];
    double dsum[BM_THREADS / 32];
  };
  BmCand top[BM_MOST_KEEP];
  float wmax[BM_THREADS / 32];
  float ref[BM_THREADS / 32], sum[BM_THREADS / 32];
  float bar;
  unsigned long long bar_key;
  BmCand bar_cand;
  unsigned long long again, done;                         // beams whose sums are computed in 64 bits; that have ended
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
      BmType<T>::unpack(row.piece(at + tid), f);
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

// log sum exp of a row in 64 bits.  2^f, |f| <= 1/2, by its Taylor polynomial of degree 11 (error below 1e-14)
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
  const double m = bm_logit(top), log2e = 1.44269504088896340735992;
  double s = 0.0;
  constexpr int N = 8;
  for (int at = tid; at < a.vocab; at += N * BM_THREADS) {
    float f[N];
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = at + i * BM_THREADS < a.vocab ? BmType<T>::load(row + at + i * BM_THREADS) : -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) s += bm_exp2(((double)fminf(f[i], BmType<T>::most) - m) * log2e);
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  __syncthreads();
  if ((tid & 31) == 0) sh.dsum[tid >> 5] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < BM_THREADS / 32; ++w) s += sh.dsum[w];
  return m + log(s);
}

// The candidates of a group: its beams' lists, an ended beam's one.  Whole block of the CTA that arrived last.
template <typename T>
__device__ __noinline__ void bm_join(BmShared& sh, const BmArgs& a, int group) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = a.beams, K = a.keep;
  const int per_beam = a.splits * K, total = B * per_beam;
  const unsigned long long* keys = a.keys + (size_t)group * B * per_beam;
  const float2* sums = a.sums + (size_t)group * B * a.splits;
  const float* scores = a.scores + (size_t)group * B;
  const uint8_t* ended = a.ended ? a.ended + (size_t)group * B : nullptr;
  // asked for early
  const unsigned long long first_key = tid < total ? __ldcg(keys + tid) : 0;
  if (tid == 0) sh.done = 0;
  __syncthreads();
  for (int b = warp; b < B; b += BM_THREADS / 32) {
    const float score = __ldcg(scores + b);
    const bool done = ended && __ldcg(ended + b);
    double c = bm_live(score) ? (double)score : -INFINITY, lse = 0.0;
    if (done && lane == 0) atomicOr(&sh.done, 1ull << b);
    if (bm_live(score) && !done) {
      float m = -INFINITY;
      for (int s = lane; s < a.splits; s += 32) {
        const float2 x = __ldcg(sums + b * a.splits + s);
        if (x.y > 0.f) m = fmaxf(m, x.x);
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      double sum = 0.0;
      for (int s = lane; s < a.splits; s += 32) {
        const float2 x = __ldcg(sums + b * a.splits + s);
        if (x.y > 0.f) sum += (double)x.y * bm_exp2(((double)x.x - (double)m) * 1.44269504088896340735992);
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (sum > 0.0) lse = (double)m + log(sum);
      else c = -INFINITY;
    }
    if (lane == 0) {
      sh.j.score[b] = c;
      sh.j.lse[b] = lse;
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
      if (i == b * per_beam && a.end_token >= 0) x = {bm_order(c), (unsigned long long)b << 32 | (uint32_t)a.end_token};
      return x;
    }
    if (key) x = {bm_order(c + ((double)bm_logit(key) - sh.j.lse[b])), (unsigned long long)b << 32 | (uint32_t)bm_token(key)};
    return x;
  };
  auto both_done = [&](const BmCand& x, const BmCand& y) { return sh.done >> (x.at >> 32) & sh.done >> (y.at >> 32) & 1; };   // no sums in them
  auto differ = [&](const BmCand& x, const BmCand& y) {   // two neighbours whose order the errors of the sums could change
    if (bm_value(x.v) - bm_value(y.v) <= kClose && x.at >> 32 != y.at >> 32 && !both_done(x, y))
      atomicOr(&sh.again, 1ull << (x.at >> 32) | 1ull << (y.at >> 32));
  };

  for (bool refined = false;; refined = true) {
    if (tid == 0) sh.count = 0;
    __syncthreads();
    long long bar = kNoCand + 1;
    const bool direct = total <= BM_DIRECT;               // every candidate is compared with every other
    if (!direct) {
      // the bar: the keep-th of the threads' best ones, less what the errors of the sums could change
      BmCand best = {kNoCand, ~0ull};
      for (int i = tid; i < total; i += BM_THREADS) {
        const BmCand x = cand(i, __ldcg(keys + i));
        if (bm_before(x, best)) best = x;
      }
      sh.most[tid] = best;
      if (tid == 0) sh.bar_cand.v = bar;
      __syncthreads();
      if (best.at != ~0ull) {
        int larger = 0;
        for (int i = 0; i < BM_THREADS; ++i) larger += bm_before(sh.most[i], best);
        if (larger == K - 1) sh.bar_cand.v = bm_order(bm_value(best.v) - kClose);
      }
      __syncthreads();
      bar = sh.bar_cand.v;
    }
    for (int i = tid; i < total; i += BM_THREADS) {
      const BmCand x = cand(i, direct && i == tid ? first_key : __ldcg(keys + i));
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
      for (int i = tid; i < count; i += BM_THREADS) {
        const BmCand x = sh.j.cand[i];
        int rank = 0;
        for (int k = 0; k < count; ++k) rank += bm_before(sh.j.cand[k], x);
        if (rank < K) sh.top[rank] = x;
      }
      __syncthreads();
      if (!refined) {
        for (int i = tid; i + 1 < found; i += BM_THREADS) differ(sh.top[i], sh.top[i + 1]);
        if (count > K) {                                  // and those that could come in
          const BmCand x = sh.top[K - 1];
          for (int i = tid; i < count; i += BM_THREADS)
            if (bm_before(x, sh.j.cand[i])) differ(x, sh.j.cand[i]);
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
          const BmCand y = cand(i, __ldcg(keys + i));
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
        const unsigned long long at = some ? sh.top[i].at : 0;
        const size_t o = (size_t)group * K + i;
        const int token = some ? (int)(uint32_t)at : -1;
        a.out_scores[o] = some ? (float)bm_value(sh.top[i].v) : -INFINITY;
        a.out_tokens[o] = token;
        a.out_parents[o] = group * B + (some ? (int)(at >> 32) : min(i, B - 1));
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
__global__ void __launch_bounds__(BM_THREADS, 4) beam_select_kernel(BmArgs a) {
  constexpr int N = BmType<T>::N;
  __shared__ BmShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x / a.splits, split = blockIdx.x - r * a.splits, group = r / a.beams;
  const BmRow<T> row(a, r);
  const int p0 = min(row.pieces, split * a.per), p1 = min(row.pieces, p0 + a.per);
  const bool front = split == 0, back = split == a.splits - 1;
  uint4 w[BM_UNROLL];
  auto load = [&](int at) {
#pragma unroll
    for (int u = 0; u < BM_UNROLL; ++u) {
      const int i = at + u * BM_THREADS + tid;
      if (i < p1) w[u] = row.piece(i);
    }
  };
  pg_wait();
  // the first tile is asked for before it is known whether the beam takes part
  const float score = __ldcg(a.scores + r);
  const bool done = a.ended && __ldcg(a.ended + r);
  load(p0);
  const int single = row.single(tid, front, back);
  const float lone = single >= 0 ? fminf(BmType<T>::load(row.base + single), BmType<T>::most) : -INFINITY;
  if (bm_live(score) && !done) {
    unsigned long long* out = a.keys + ((size_t)r * a.splits + split) * a.keep;

    // ---- the first tile: reference and bar ----
    float best = lone;
#pragma unroll
    for (int u = 0; u < BM_UNROLL; ++u) {
      if (p0 + u * BM_THREADS + tid < p1) {
        float f[N];
        BmType<T>::unpack(w[u], f);
#pragma unroll
        for (int i = 0; i < N; ++i) best = fmaxf(best, f[i]);
      }
    }
    best = fminf(best, BmType<T>::most);
    float ref = fmaxf(bm_block_max(sh, best), -FLT_MAX);
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
    const float bar = fmaxf(sh.bar, -FLT_MAX);            // -inf is no candidate

    // ---- the stretch ----
    float limit = ref + kRefFar;
    uint64_t sum2 = 0;                                    // of a tile
    double sum = 0.0;
    auto push = [&](float l, int token) {
      const int n = atomicAdd(&sh.count, 1);
      if (n < BM_LIST) sh.list[n] = bm_key(l, token);
    };
    if (lone >= bar) push(lone, single);
    if (lone > -INFINITY) sum = pa_ex2((lone - ref) * 1.4426950408889634f);
    for (int at = p0; at < p1; at += BM_TILE) {
      uint4 v[BM_UNROLL];
#pragma unroll
      for (int u = 0; u < BM_UNROLL; ++u) v[u] = w[u];
      load(at + BM_TILE);
#pragma unroll
      for (int u = 0; u < BM_UNROLL; ++u) {
        const int i = at + u * BM_THREADS + tid;
        if (i >= p1) break;
        float f[N];
        BmType<T>::unpack(v[u], f);
        float most = f[0];
#pragma unroll
        for (int e = 1; e < N; ++e) most = fmaxf(most, f[e]);
        if (most > limit) {
#pragma unroll
          for (int e = 0; e < N; ++e) f[e] = fminf(f[e], BmType<T>::most);
          most = fminf(most, BmType<T>::most);
          if (most > ref) {
            float s0, s1;
            f32x2_unpack(sum2, s0, s1);
            sum = (sum + (double)(s0 + s1)) * (double)pa_ex2((ref - most) * 1.4426950408889634f);
            sum2 = 0;
            ref = most;
            limit = ref + kRefFar;
          }
        }
        const uint64_t back2 = f32x2_pack(-ref, -ref), scale2 = f32x2_pack(1.4426950408889634f, 1.4426950408889634f);
        uint64_t part = 0;
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          float x0, x1;
          f32x2_unpack(f32x2_mul(f32x2_add(f32x2_pack(f[e], f[e + 1]), back2), scale2), x0, x1);
          part = f32x2_add(part, f32x2_pack(pa_ex2(x0), pa_ex2(x1)));
        }
        sum2 = f32x2_add(sum2, part);
        if (most >= bar) {
          const int token = row.token(i);
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (f[e] >= bar) push(f[e], token + e);
        }
      }
      float s0, s1;
      f32x2_unpack(sum2, s0, s1);
      sum += (double)(s0 + s1);
      sum2 = 0;
    }
    // ---- its sum and its largest ----
    const float high = bm_block_max(sh, ref);
    double all = sum * (ref == high ? 1.0 : (double)pa_ex2((ref - high) * 1.4426950408889634f));
#pragma unroll
    for (int d = 16; d; d >>= 1) all += __shfl_xor_sync(0xffffffffu, all, d);
    if (lane == 0) sh.dsum[warp] = all;
    __syncthreads();
    if (tid == 0) {
      all = 0.0;
      for (int i = 0; i < BM_THREADS / 32; ++i) all += sh.dsum[i];
      a.sums[(size_t)r * a.splits + split] = make_float2(high, (float)all);
    }
    const int count = sh.count;
    if (count > BM_LIST) {
      bm_crowded<T>(sh, a, row, p0, p1, front, back, out);
    } else {
      for (int i = tid; i < count; i += BM_THREADS) {
        const unsigned long long mine = sh.list[i];
        int rank = 0;
        for (int k = 0; k < count; ++k) rank += sh.list[k] > mine;
        if (rank < a.keep) out[rank] = mine;
      }
      for (int i = count + tid; i < a.keep; i += BM_THREADS) out[i] = 0;
    }
  }
  // ---- the last CTA of the group joins ----
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    const int n = a.beams * a.splits;
    sh.last = atomicAdd(a.counters + group, 1) == n - 1;
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
  int splits;
};

static bool valid_beams(const less_beams* d) {
  if (d->groups < 1 || d->beams < 1 || d->beams > BM_MOST_BEAMS || d->vocab < 1 || d->keep < 1 || d->keep > BM_MOST_KEEP) return false;
  if (d->flags & ~(uint32_t)(LESS_BEAMS_BF16 | LESS_BEAMS_F32) || d->flags == (LESS_BEAMS_BF16 | LESS_BEAMS_F32)) return false;
  if (d->end_token < -1 || d->end_token >= d->vocab) return false;
  return d->groups <= (1 << 20) / d->beams;               // rows
}

// A row is cut so that all CTAs of a call, four on a multiprocessor, run at once, but for no less than 4096 elements each, nor
// into so many lists that joining them shows (64 groups of 8 beams of 128 256: cut in five, 4.3 times as many, 77 us).
static BmLayout bm_layout(const less_beams* d) {
  BmLayout l;
  const int64_t rows = (int64_t)d->groups * d->beams;
  int64_t s = pg_ceil(d->vocab, 4096);
  if (s > 4 * 148 / rows) s = 4 * 148 / rows;
  if (s > BM_JOINED / (d->beams * d->keep)) s = BM_JOINED / (d->beams * d->keep);
  l.splits = (int)(s < 1 ? 1 : s);
  size_t at = ((size_t)d->groups * 4 + 255) / 256 * 256;
  l.sums = at;
  at = (at + (size_t)rows * l.splits * 8 + 255) / 256 * 256;
  l.keys = at;
  l.total = (at + (size_t)rows * l.splits * d->keep * 8 + 255) / 256 * 256;
  return l;
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
  const int pieces = (int)(((int64_t)d->vocab * size + 15) / 16);
  BmArgs a = {logits, row_stride, scores, ended, d->groups, d->beams, d->vocab, d->keep, d->end_token, l.splits,
              (pieces + l.splits - 1) / l.splits, out_scores, out_tokens, out_parents, out_ended, (int32_t*)w, (float2*)(w + l.sums),
              (unsigned long long*)(w + l.keys)};
  const dim3 grid((unsigned)(d->groups * d->beams * l.splits));
  cudaStream_t s = (cudaStream_t)stream;
  if (d->flags & LESS_BEAMS_F32) return pg_launch("beam_select_kernel", beam_select_kernel<float>, grid, BM_THREADS, 0, s, a);
  if (d->flags & LESS_BEAMS_BF16) return pg_launch("beam_select_kernel", beam_select_kernel<__nv_bfloat16>, grid, BM_THREADS, 0, s, a);
  return pg_launch("beam_select_kernel", beam_select_kernel<__half>, grid, BM_THREADS, 0, s, a);
}
