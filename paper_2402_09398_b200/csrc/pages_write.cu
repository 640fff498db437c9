// The write of the paged 8-bit cache: the new tokens of every sequence, rounded to 8 bits.
//
//   a = max |x| over the 16 tokens x D dimensions of a block (with the magnitude it had, if it holds older tokens)
//   code = rn(x * top / a)            top = 127 (int8) or 448 (e4m3), ties to even
//   older tokens of the block, where a has grown:  code = rn(code * a_old / a)
//
// The codes are those of exact arithmetic, without a division per value.  A 16-bit value (an old code, exactly) times the
// correctly rounded top / a (a_old / a) is off by at most 2^-23 relative.  A quotient that is not a tie is at least 2^-19
// from the nearest one (both are ratios of integers of at most 8 + 11 bits), so rounding to 21 bits first (2^-21) lands
// ties exactly on themselves and nothing else on a tie; the second rounding is then right.  (Magnitudes of more bits, which
// only a cache that its owner has filled can have, go another way: pw_foreign_block.)
// Infinities are written as the largest finite fp16 number (bf16: 2^100, so that x * top stays finite), NaN as 0:
// one bad token must not take the other fifteen of its block with it.  Magnitudes below 2^-100 (bf16) become 0: the
// attention divides by magnitudes.  Tokens of the last block behind the
// sequence's end get code 0.
//
// Bound by memory: 2 bytes read and 1 written per value.  A block of threads takes one 16-token block of one layer
// for a few heads; a thread owns one 16-byte piece of the stored tile (pages.cuh), so the stores are contiguous.
// Measured: 18 400 tokens of four layers, 8 heads of D 128 (452 MB): 116 us, 3.9 TB/s of 6.5; with a division per value
// 376, one head ahead 158, fp32 maxima 145.  The rest is the chain per head: loads, maximum over 4 warps, stores.
#include <type_traits>

#include "less_internal.cuh"
#include "pages.cuh"

namespace less {

constexpr int PW_THREADS = 256;

struct PwArgs {
  const void* k;
  const void* v;
  int64_t k_stride, v_stride;        // elements from token to token
  const int32_t* seqs;
  const int32_t* starts;
  int n, rows, layer0;
  bool marked;                       // mark holds the first entry of every listed sequence
};

// Lists of more entries than PW_LOOK: the first entry of every sequence goes to mark, in two launches.  Up to that an entry
// looks through those before it, which is as many loads as there are pairs of them.  Measured, looking / marking, one token
// each of one layer, 8 heads: 64 entries 4.9 / 6.4 us, 2048 32.0 / 32.0, 4096 66.9 / 63.4, 65 536 3450 / 887.
constexpr int PW_LOOK = 2048;
template <bool INIT>
__global__ void __launch_bounds__(PW_THREADS) pages_mark_kernel(PgParams p, const int32_t* seqs, int n) {
  pg_wait();
  for (int64_t i = (int64_t)blockIdx.x * PW_THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * PW_THREADS) {
    const int s = __ldg(seqs + i);
    if (s < 0 || s >= p.seqs) continue;
    if (INIT) p.mark[s] = n;
    else atomicMin(p.mark + s, (int)i);
  }
}

// block slots of a call: entry i owns slots [starts[i] / 16 + 2 i, starts[i + 1] / 16 + 2 (i + 1)) - at least as many
// as its `count` tokens can touch, (count + 14) / 16 + 1, whatever their first position is
__device__ __forceinline__ int pw_slot(const PwArgs& a, int i) {
  const int row = a.starts ? min(max(__ldg(a.starts + i), 0), a.rows) : i;
  return row / kPageBlock + 2 * i;
}

template <typename T>
__device__ __forceinline__ float pw_load(T x) {
  constexpr float most = std::is_same<T, __half>::value ? 65504.f : 0x1p100f;
  const float f = static_cast<float>(x);
  return f == f ? fminf(fmaxf(f, -most), most) : 0.f;
}

template <bool E4M3>
__device__ __forceinline__ float pw_value(uint32_t code) {   // in units of amax / top
  if (E4M3) {
    const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3);
    return __half2float(__half(h));
  }
  return (float)(int8_t)code;
}

// four values times a factor -> four codes
template <bool E4M3>
__device__ __forceinline__ uint32_t pw_codes(float x0, float x1, float x2, float x3, float factor) {
  const uint64_t f = f32x2_pack(factor, factor), nine = f32x2_pack(9.f, 9.f), minus = f32x2_pack(-1.f, -1.f);
  uint64_t y[2] = {f32x2_mul(f32x2_pack(x0, x1), f), f32x2_mul(f32x2_pack(x2, x3), f)};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint64_t c = f32x2_mul(y[i], nine);            // 2^3 + 1: c - (c - y) is y to 21 bits
    y[i] = f32x2_fma(f32x2_fma(y[i], minus, c), minus, c);
  }
  float a, b, c, d;
  if (E4M3) {
    f32x2_unpack(y[0], a, b);
    f32x2_unpack(y[1], c, d);
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
  }
  // + 1.5 * 2^23 rounds to an integer, whose low byte is the code
  const uint64_t one = f32x2_pack(1.f, 1.f), magic = f32x2_pack(12582912.f, 12582912.f);
  f32x2_unpack(f32x2_fma(y[0], one, magic), a, b);
  f32x2_unpack(f32x2_fma(y[1], one, magic), c, d);
  return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040),
                     __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
}

// The same where a magnitude is not one of the 16-bit inputs' (a cache that the caller has filled): the quotient
// value * num / m may then lie nearer to a tie than fp32 can tell.  y, to 21 bits, is a tie exactly or far from one; the
// sign of value * num - y * m, which 64 bits hold exactly, says on which side of it the quotient is.
__device__ __forceinline__ bool pw_foreign(float m) { return (__float_as_uint(m) & 0x1fffu) != 0; }   // more than 11 bits
__device__ __forceinline__ float pw_beside(float x, float num, float m) {
  const float q = __fdiv_rn(num, m) * x, c = __fmul_rn(q, 9.f), y = c - __fadd_rn(c, -q);
  const double d = fma((double)x, (double)num, -(double)y * (double)m);
  if (y == 0.f || d == 0.) return y;
  return __int_as_float(__float_as_int(y) + ((d > 0.) == (y > 0.f) ? 1 : -1));
}
template <bool E4M3>
__device__ __forceinline__ uint32_t pw_code_foreign(float x, float num, float m) {
  const float y = pw_beside(x, num, m);
  return E4M3 ? __nv_cvt_float_to_fp8(y, __NV_SATFINITE, __NV_E4M3) : (uint32_t)__float2int_rn(y) & 0xffu;
}

// two packed 16-bit values -> fp32
template <typename T>
__device__ __forceinline__ void pw_pair(uint32_t u, float& a, float& b);
template <>
__device__ __forceinline__ void pw_pair<__half>(uint32_t u, float& a, float& b) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
  a = f.x;
  b = f.y;
}
template <>
__device__ __forceinline__ void pw_pair<__nv_bfloat16>(uint32_t u, float& a, float& b) {
  a = __uint_as_float(u << 16);
  b = __uint_as_float(u & 0xffff0000u);
}
// the largest finite value of pw_load, as bits: 65504, 2^100
template <typename T>
__device__ __forceinline__ constexpr uint32_t pw_most_bits() { return std::is_same<T, __half>::value ? 0x7bffu : 0x7180u; }
template <typename T>
__device__ __forceinline__ uint32_t pw_clean(uint32_t u) {                // two values, each as pw_load takes it
  T v[2];
  *reinterpret_cast<uint32_t*>(v) = u;
  v[0] = T(pw_load(v[0]));
  v[1] = T(pw_load(v[1]));
  return *reinterpret_cast<uint32_t*>(v);
}

// byte of (token, dimension) in a tile of keys or values (pages.cuh)
template <int D>
__device__ __forceinline__ int pw_byte(int which, int token, int d) {
  const int c = which ? d % (D / 8) / 4 : (token >> 1 & 1) * (D / 64) + d % (D / 4) / 16;
  const int g = which ? d / (D / 8) : 2 * (token >> 2) + (token & 1), t = which ? token >> 2 : d / (D / 4);
  return (32 * c + 4 * g + t) * 16 + (which ? d % 4 * 4 + (token & 3) : d % 16);
}
// The keys or values of one block of one head, whatever the older magnitude is: by one warp, a byte at a time.  `src`: the
// first of live - keep new tokens.
template <typename T, int D, bool E4M3>
__device__ __noinline__ void pw_foreign_block(const T* src, int64_t stride, int which, int keep, int live, uint8_t* tile, float* mag) {
  const int lane = threadIdx.x & 31;
  const float old = keep > 0 ? __ldcg(mag) : 0.f;
  uint32_t most = 0;
  for (int i = lane; i < (live - keep) * D; i += 32)
    most = max(most, __float_as_uint(fabsf(pw_load(src[(int64_t)(i / D) * stride + i % D]))));
  float m = fmaxf(__uint_as_float(__reduce_max_sync(0xffffffffu, most)), old);
  if (m < 0x1p-100f) m = 0.f;
  const float unit = m > 0.f ? m : 1.f;
  for (int i = lane; i < kPageBlock * D; i += 32) {
    const int token = i / D, d = i % D;
    uint8_t* at = tile + pw_byte<D>(which, token, d);
    uint32_t code = 0;
    if (token < keep) {
      code = __ldcg(at);
      if (m != old) code = pw_code_foreign<E4M3>(pw_value<E4M3>(code), old, unit);
    } else if (token < live) {
      code = pw_code_foreign<E4M3>(pw_load(src[(int64_t)(token - keep) * stride + d]), pg_top<E4M3>(), unit);
    }
    *at = (uint8_t)code;
  }
  __syncwarp();                                          // all lanes have read the older magnitude
  if (lane == 0) *mag = m;
}

template <typename T, int D, bool E4M3>
__global__ void __launch_bounds__(PW_THREADS, 4) pages_write_kernel(PgParams p, PwArgs a) {
  constexpr int PER = D;                        // threads per (head, keys or values): one 16-byte piece each
  constexpr int HEADS = PW_THREADS / (2 * PER); // heads per turn
  __shared__ uint32_t red[2][PW_THREADS / 32];
  const int tid = threadIdx.x, lane = tid & 31;
  pg_wait();
  bool again = __ldcg(p.status) != 0;           // nothing after an error of an earlier call
  p.status += kLateStatus;
  const int slot = blockIdx.x;
  if (slot == (int)gridDim.x - 1) {             // one CTA more than there are slots
    pg_check_starts(p, a.starts, a.n);
    return;
  }
  int lo = 0, hi = a.n - 1;                     // the last entry whose slots start at or before this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pw_slot(a, mid) <= slot) lo = mid; else hi = mid - 1;
  }
  const PgEntry e = pg_entry(p, a.seqs, a.starts, a.rows, lo);
  const int begin = e.len - e.count;            // first new position
  const int first = pw_slot(a, lo);
  if (e.count == 0 || slot < first) return;     // slots before the first entry's: its rows need not start at 0
  if (begin < 0) {
    if (tid == 0) pg_status(p.status, kPagesBounds, 40);
    return;
  }
  const int64_t block = begin / kPageBlock + (int64_t)(slot - first);
  if (block * kPageBlock >= e.len) return;
  const int pos0 = (int)block * kPageBlock;
  const int keep = begin - pos0;                         // tokens of the block older than the call (<= 0: none)
  const int live = min(kPageBlock, e.len - pos0);
  const int lj = blockIdx.z, layer = a.layer0 + lj;
  // Which piece is whose: of the keys in stored order (a thread's 16 values are 32 bytes of one row), of the values such
  // that neighbouring threads have neighbouring dimensions (four rows' 8 bytes each: whole sectors per warp)
  const int which = (tid / PER) & 1, own = tid % PER;
  const int c = which ? own % (D / 32) : own >> 5, t = which ? own / (D / 32) % 4 : own & 3, g = which ? own / (D / 8) : (own >> 2) & 7;
  const int piece = 32 * c + 4 * g + t;
  const int token = 4 * (g >> 1) + 2 * (c / (D / 64)) + (g & 1);       // of a piece of keys

  // a head's 16 new values of this thread, as they come
  const int64_t stride = which ? a.v_stride : a.k_stride;
  const T* src = reinterpret_cast<const T*>(which ? a.v : a.k) + (int64_t)(e.row0 - keep) * stride + (int64_t)lj * p.heads * D;
  src += which ? (int64_t)(4 * t) * stride + g * (D / 8) + c * 4 : (int64_t)token * stride + t * (D / 4) + (c % (D / 64)) * 16;
  auto fetch = [&](int h, uint2 (&raw)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) raw[k] = make_uint2(0, 0);
    if (h >= p.heads) return;
    const T* s = src + (int64_t)h * D;
    if (which == 0) {
      if (token >= keep && token < live) {
        const uint4 x = __ldg(reinterpret_cast<const uint4*>(s)), y = __ldg(reinterpret_cast<const uint4*>(s) + 1);
        raw[0] = make_uint2(x.x, x.y);
        raw[1] = make_uint2(x.z, x.w);
        raw[2] = make_uint2(y.x, y.y);
        raw[3] = make_uint2(y.z, y.w);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (4 * t + k >= keep && 4 * t + k < live) raw[k] = __ldcs(reinterpret_cast<const uint2*>(s + (int64_t)k * stride));
    }
  };
  // two heads on their way beside the one that is worked on: 4 CTAs x 16 KB per SM
  uint2 raw[4], ahead[2][4];
  const int h_first = (int)blockIdx.y * HEADS + tid / (2 * PER), h_step = (int)gridDim.y * HEADS;
  fetch(h_first, raw);
  fetch(h_first + h_step, ahead[0]);

  // a sequence listed twice: the first entry counts
  if (a.marked) again |= __ldcg(p.mark + e.seq) != lo;
  else
    for (int j = tid; j < lo; j += PW_THREADS) again |= __ldg(a.seqs + j) == e.seq;
  const int page = pg_page(p, e.seq, pos0 >> p.pt_shift);
  const int refs = page >= 0 ? __ldcg(p.refs + page) : 0;
  if (__syncthreads_or(again)) return;
  if (refs != 1) {                                       // trimmed, or held by other sequences too
    if (tid == 0) pg_status(p.status, page < 0 ? kPagesBounds : kPagesState, 41);
    return;
  }
  const int inner = (pos0 & (p.pt - 1)) / kPageBlock;

  if (keep > 0) {
    // Older magnitudes are looked at before the loop, whose registers the other way would take (prompts: 135 us against 116)
    auto head_of = [&](int i) { return ((int)blockIdx.y + i / HEADS * (int)gridDim.y) * HEADS + i % HEADS; };   // i-th of the CTA
    bool foreign = false;
    for (int i = tid; head_of(i >> 1) < p.heads; i += PW_THREADS)
      foreign |= pw_foreign(__ldcg(p.amax + pg_mag(p, layer, page, head_of(i >> 1)) + (i & 1) * (p.pt / kPageBlock) + inner));
    if (__syncthreads_or(foreign)) {
      for (int i = tid >> 5; head_of(i >> 1) < p.heads; i += PW_THREADS / 32) {
        const int h = head_of(i >> 1), kv = i & 1;
        const int64_t step = kv ? a.v_stride : a.k_stride;
        pw_foreign_block<T, D, E4M3>(reinterpret_cast<const T*>(kv ? a.v : a.k) + e.row0 * step + ((int64_t)lj * p.heads + h) * D, step, kv, keep, live,
                                     p.codes + pg_slab(p, D, layer, page, h) + ((size_t)kv * p.pt + inner * kPageBlock) * D,
                                     p.amax + pg_mag(p, layer, page, h) + kv * (p.pt / kPageBlock) + inner);
      }
      return;
    }
  }

  int turn = 0;
  for (int h0 = (int)blockIdx.y * HEADS; h0 < p.heads; h0 += h_step, turn ^= 1) {
    const int h = h0 + tid / (2 * PER);
    const bool in = h < p.heads;
    fetch(h + 2 * h_step, ahead[1]);
    uint8_t* tile = p.codes + pg_slab(p, D, layer, page, in ? h : 0) + ((size_t)which * p.pt + inner * kPageBlock) * D + piece * 16;
    float* mag = p.amax + pg_mag(p, layer, page, in ? h : 0) + which * (p.pt / kPageBlock) + inner;
    uint4 was = make_uint4(0, 0, 0, 0);
    float old = 0.f;
    if (in && keep > 0) {
      was = __ldcg(reinterpret_cast<const uint4*>(tile));
      old = __ldcg(mag);
    }
    // the largest magnitude, as bits (not negative: their order is that of the bits); what is not finite is rare
    uint32_t* word = reinterpret_cast<uint32_t*>(raw);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = __vmaxu2(most, word[i] & 0x7fff7fffu);
    most = max(most >> 16, most & 0xffffu);
    if (most > pw_most_bits<T>()) {
      most = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        word[i] = pw_clean<T>(word[i]);
        most = __vmaxu2(most, word[i] & 0x7fff7fffu);
      }
      most = max(most >> 16, most & 0xffffu);
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) red[turn][tid >> 5] = most;
    __syncthreads();                                     // the other half of red is free: it was read a turn ago
    most = 0;
#pragma unroll
    for (int w = 0; w < PER / 32; ++w) most = max(most, red[turn][tid / PER * (PER / 32) + w]);
    float m, unused;
    pw_pair<T>(most, m, unused);
    m = fmaxf(m, old);
    if (m < 0x1p-100f) m = 0.f;                          // its codes come out as 0 too
    if (in) {
      const float unit = m > 0.f ? m : 1.f, factor = __fdiv_rn(pg_top<E4M3>(), unit);
      float x[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) pw_pair<T>(word[i], x[2 * i], x[2 * i + 1]);
      uint32_t out[4];
      if (which == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = pw_codes<E4M3>(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3], factor);
      } else {                                           // token by token they came, a word is one dimension, four tokens
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = pw_codes<E4M3>(x[i], x[4 + i], x[8 + i], x[12 + i], factor);
      }
      if (keep > 0) {
        // of a word's four codes, those of older tokens: of the keys all or none, of the values the first few
        const int older = which ? min(max(keep - 4 * t, 0), 4) : token < keep ? 4 : 0;
        const uint32_t mask = older == 4 ? 0xffffffffu : (1u << (8 * older)) - 1;
        const float again = __fdiv_rn(old, unit);
        const uint32_t ww[4] = {was.x, was.y, was.z, was.w};
        if (older)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t w = ww[i] & mask;
            if (m != old)
              w = pw_codes<E4M3>(pw_value<E4M3>(w & 0xffu), pw_value<E4M3>(w >> 8 & 0xffu), pw_value<E4M3>(w >> 16 & 0xffu),
                                 pw_value<E4M3>(w >> 24), again);
            out[i] = (out[i] & ~mask) | (w & mask);
          }
      }
      *reinterpret_cast<uint4*>(tile) = make_uint4(out[0], out[1], out[2], out[3]);
      if (own == 0) *mag = m;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      raw[k] = ahead[0][k];
      ahead[0][k] = ahead[1][k];
    }
  }
}

// One new token per sequence, a warp per (sequence, layer, head), which puts both tiles of the block back: older tokens
// as they were or, if the magnitude has grown, rounded again, zeros behind the end, and then the token's own codes (a
// lane's four dimensions of the keys are four neighbouring bytes, those of the values lie four bytes apart).  What counts
// is the chain of loads that leads to the tiles: all that does not depend on one another is asked for at once.
// Measured: 64 sequences, four layers, 8 heads, resize before it: 10 us replayed, launches included; 0.2 us of memory traffic.
template <typename T, int D, bool E4M3>
__global__ void __launch_bounds__(PW_THREADS) pages_write_one_kernel(PgParams p, PwArgs a, int nl) {
  constexpr int PL = D / 32, PIECES = D / 32;   // values of a lane; 16-byte pieces of a lane in a tile
  const int lane = threadIdx.x & 31;
  pg_wait();
  const int64_t w = (int64_t)blockIdx.x * (PW_THREADS / 32) + (threadIdx.x >> 5);
  const int per = nl * p.heads, i = (int)(w / per), rest = (int)(w - (int64_t)i * per), lj = rest / p.heads, h = rest - lj * p.heads;
  if (i >= a.n) return;
  T raw[2][PL];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const T* src = reinterpret_cast<const T*>(which ? a.v : a.k) + (int64_t)i * (which ? a.v_stride : a.k_stride) +
                   (int64_t)(lj * p.heads + h) * D + lane * PL;
    if (PL == 4) *reinterpret_cast<uint2*>(raw[which]) = __ldcs(reinterpret_cast<const uint2*>(src));
    else *reinterpret_cast<uint32_t*>(raw[which]) = __ldcs(reinterpret_cast<const uint32_t*>(src));
  }
  bool again = __ldcg(p.status) != 0;
  p.status += kLateStatus;
  const PgEntry e = pg_entry(p, a.seqs, nullptr, a.rows, i);
  if (a.marked) again |= __ldcg(p.mark + e.seq) != i;
  else
    for (int j = lane; j < i; j += 32) again |= __ldg(a.seqs + j) == e.seq;
  if (e.count == 0) return;
  if (e.len == 0) {
    if (lane == 0) pg_status(p.status, kPagesBounds, 42);
    return;
  }
  const int pos = e.len - 1, page = pg_page(p, e.seq, pos >> p.pt_shift);
  if (__any_sync(0xffffffffu, again)) return;
  if (page < 0 || __ldcg(p.refs + page) != 1) {          // trimmed, or held by other sequences too
    if (lane == 0) pg_status(p.status, page < 0 ? kPagesBounds : kPagesState, 43);
    return;
  }
  const int inner = (pos & (p.pt - 1)) / kPageBlock, token = pos % kPageBlock, layer = a.layer0 + lj;
  float* mags = p.amax + pg_mag(p, layer, page, h) + inner;
  uint8_t* tiles = p.codes + pg_slab(p, D, layer, page, h) + (size_t)inner * kPageBlock * D;
  float old[2] = {0.f, 0.f};
  uint4 was[2][PIECES];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (token) old[which] = __ldcg(mags + which * (p.pt / kPageBlock));
#pragma unroll
    for (int c = 0; c < PIECES; ++c)
      was[which][c] = token ? __ldcg(reinterpret_cast<const uint4*>(tiles + (size_t)which * p.pt * D + c * 512 + lane * 16)) : make_uint4(0, 0, 0, 0);
  }
  if (pw_foreign(old[0]) || pw_foreign(old[1])) {
    for (int which = 0; which < 2; ++which) {
      const int64_t stride = which ? a.v_stride : a.k_stride;
      pw_foreign_block<T, D, E4M3>(reinterpret_cast<const T*>(which ? a.v : a.k) + (int64_t)i * stride + (int64_t)(lj * p.heads + h) * D, stride,
                                   which, token, token + 1, tiles + (size_t)which * p.pt * D, mags + which * (p.pt / kPageBlock));
    }
    return;
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    uint8_t* tile = tiles + (size_t)which * p.pt * D;
    float x[4] = {0.f, 0.f, 0.f, 0.f}, m = 0.f;
#pragma unroll
    for (int k = 0; k < PL; ++k) {
      x[k] = pw_load(raw[which][k]);
      m = fmaxf(m, fabsf(x[k]));
    }
    // magnitudes are not negative: their order is that of their bits
    m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
    m = fmaxf(m, old[which]);
    if (m < 0x1p-100f) m = 0.f;
    const float unit = m > 0.f ? m : 1.f, factor = __fdiv_rn(old[which], unit);
    const uint32_t mine = pw_codes<E4M3>(x[0], x[1], x[2], x[3], __fdiv_rn(pg_top<E4M3>(), unit));
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int c = 0; c < PIECES; ++c) {
      // which of a word's four codes are older tokens': of the keys all or none, of the values the first few
      const int row = 4 * (g >> 1) + 2 * (c / (D / 64)) + (g & 1), older = which ? min(max(token - 4 * t, 0), 4) : row < token ? 4 : 0;
      const uint32_t keep = older == 4 ? 0xffffffffu : (1u << (8 * older)) - 1;
      const uint32_t w[4] = {was[which][c].x & keep, was[which][c].y & keep, was[which][c].z & keep, was[which][c].w & keep};
      uint4 out = make_uint4(w[0], w[1], w[2], w[3]);
      if (m != old[which]) {
        uint32_t again[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float y[4];
#pragma unroll
          for (int b = 0; b < 4; ++b) y[b] = b < older ? pw_value<E4M3>((w[q] >> (8 * b)) & 0xffu) : 0.f;
          again[q] = pw_codes<E4M3>(y[0], y[1], y[2], y[3], factor);
        }
        out = make_uint4(again[0], again[1], again[2], again[3]);
      }
      *reinterpret_cast<uint4*>(tile + c * 512 + lane * 16) = out;
    }
    if (lane == 0 && (m != old[which] || token == 0)) mags[which * (p.pt / kPageBlock)] = m;
    __syncwarp();                                        // the token's codes go on top, from other lanes
    // the token's codes: dimensions lane * PL ..
    const int d = lane * PL;
    if (which == 0) {
      const int gk = 2 * (token >> 2) + (token & 1), j = token >> 1 & 1, tk = d / (D / 4), r = d % (D / 4);
      uint8_t* at = tile + (32 * (j * (D / 64) + r / 16) + 4 * gk + tk) * 16 + r % 16;
      if (PL == 4) *reinterpret_cast<uint32_t*>(at) = mine;
      else *reinterpret_cast<uint16_t*>(at) = (uint16_t)mine;
    } else {
      const int gv = d / (D / 8), r = d % (D / 8);
      uint8_t* at = tile + (32 * (r / 4) + 4 * gv + (token >> 2)) * 16 + (r % 4) * 4 + (token & 3);
#pragma unroll
      for (int k = 0; k < PL; ++k) at[4 * k] = (uint8_t)(mine >> (8 * k));
    }
  }
}

}  // namespace less

using namespace less;

extern "C" int less_pages_write(const less_pages* d, int32_t layer_begin, int32_t layer_count, int32_t n,
                                const int32_t* seqs, const int32_t* starts, int32_t rows, const void* k,
                                int64_t k_stride, const void* v, int64_t v_stride, void* stream) {
  PgParams p;
  int rc = pg_view(d, &p);
  if (rc != LESS_OK) return rc;
  if (layer_begin < 0 || layer_count < 1 || layer_begin > d->layers - layer_count) return LESS_ERR_BAD_LAYER_RANGE;
  if (n < 0 || n > d->seqs || rows < 0 || (!starts && rows != n)) return LESS_ERR_INVALID_CONFIG;
  if (n == 0 || rows == 0) return LESS_OK;
  if (!seqs || !k || !v) return LESS_ERR_NULL_POINTER;
  if (((uintptr_t)seqs | (uintptr_t)starts) & 3) return LESS_ERR_MISALIGNED;
  const int64_t row = (int64_t)layer_count * d->heads * d->head_dim;
  if (k_stride < row || v_stride < row) return LESS_ERR_INVALID_CONFIG;
  if ((((uintptr_t)k | (uintptr_t)v) & 15) || ((k_stride | v_stride) & 7)) return LESS_ERR_MISALIGNED;
  PwArgs a = {k, v, k_stride, v_stride, seqs, starts, n, rows, layer_begin, n > PW_LOOK};
  const bool bf16 = d->flags & LESS_PAGES_BF16, e4m3 = d->flags & LESS_PAGES_E4M3;
  // Heads of a block are taken in turn by one CTA, so that what leads to its page is looked up once and the next head's
  // rows are on their way: as many as make one wave of resident CTAs (4 per multiprocessor).  Measured, one turn a CTA /
  // all heads in one / this rule, D 128, with the resize: 200 tokens of 32 heads 8.3 / 27.9 / 8.3 us; 1000 of 32
  // 17.7 / 29.5 / 13.3; four sequences of 2000, 8 heads 30.2 / 19.2 / 19.5; 18 400 tokens of four layers, 8 heads
  // 233 / 116 / 116.
  const int turns = pg_ceil(d->heads, PW_THREADS / (2 * d->head_dim)), slots = rows / kPageBlock + 2 * n;
  const int64_t wave = 4 * pg_sms(), work = (int64_t)slots * layer_count * turns;
  const int share = work > wave * turns ? turns : (int)((work + wave - 1) / wave);
  const dim3 grid(slots + 1, pg_ceil(turns, share), layer_count);
  const int64_t one = ((int64_t)n * layer_count * d->heads + PW_THREADS / 32 - 1) / (PW_THREADS / 32);
  if (grid.y > 65535 || one > 0x7fffffff) return LESS_ERR_INVALID_CONFIG;
  cudaStream_t s = (cudaStream_t)stream;
  if (a.marked) {
    const dim3 ctas(pg_ceil(n, PW_THREADS) < 2 * pg_sms() ? pg_ceil(n, PW_THREADS) : 2 * pg_sms());
    rc = pg_launch("pages_mark_kernel", pages_mark_kernel<true>, ctas, PW_THREADS, 0, s, p, seqs, n);
    if (rc == LESS_OK) rc = pg_launch("pages_mark_kernel", pages_mark_kernel<false>, ctas, PW_THREADS, 0, s, p, seqs, n);
    if (rc != LESS_OK) return rc;
  }
#define PW_LAUNCH(T, D, E)                                                                                              \
  rc = starts ? pg_launch("pages_write_kernel", pages_write_kernel<T, D, E>, grid, PW_THREADS, 0, s, p, a)               \
              : pg_launch("pages_write_one_kernel", pages_write_one_kernel<T, D, E>, dim3(one), PW_THREADS, 0, s, p, a, layer_count)
#define PW_TYPES(D)                                                                                                      \
  if (bf16) { if (e4m3) PW_LAUNCH(__nv_bfloat16, D, true); else PW_LAUNCH(__nv_bfloat16, D, false); }                    \
  else { if (e4m3) PW_LAUNCH(__half, D, true); else PW_LAUNCH(__half, D, false); }
  if (d->head_dim == 128) { PW_TYPES(128) } else { PW_TYPES(64) }
#undef PW_TYPES
#undef PW_LAUNCH
  return rc;
}
