// What the two attention kernels over the paged 8-bit cache share (pages_attn.cu, pages_chunk.cu).
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

__device__ __forceinline__ float pa_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A row's sums are relative to 2^m of the row, a reference near the largest exponent so far.  m is a whole number, so that a
// new reference changes the sums by exact powers of two.
__device__ __forceinline__ float pa_scaled(float x, float d) { return scalbnf(x, (int)fmaxf(d, -1000.f)); }   // x 2^d
__device__ __forceinline__ float pa_pow2(float d) { return pa_scaled(1.f, d); }
// The exponents of P = p a_v include log2 a_v, so that what is rounded to fp16 is relative to the largest share of the sum,
// wherever the magnitudes of other blocks lie; p itself, for the sum of the probabilities, is 2^-log2 a_v of it.
// Magnitudes lie in [2^-100, 2^100] (less counts as values of zero): that sum is kept 2^-24 times as large, from 2^-117
// of one token to 2^100 of each.
constexpr float kLeastValue = 0x1p-100f, kNoValues = -101.f, kSumBits = 24.f;

// (reference, sum) of a part of a row, the same but with the sum in [1, 2): a weight in joining the parts is then
// sum 2^(reference - largest), which is lost only if it does not count.  Beyond 2^23 references are coarser than that.
__device__ __forceinline__ float2 pa_share(float m, float sum) {
  if (sum >= 0x1p-126f && sum < INFINITY && fabsf(m) < 0x1p23f) {
    const int bits = __float_as_int(sum);
    m += (float)((bits >> 23) - 127);
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
//   24 rows (one KV head, D 64): 16 sequences of 1000: 27 / 14 us
//   32 rows:  one of 500: 17 / 20 us; one of 2000: 31 / 21; four of 1000: 32 / 21; 64 of 100: 27 / 44;
//             128 of 2000: 280 / 294; 64 of 1000, 32 KV heads x 1: 289 / 344
//   48 rows:  two of 30 000: 111 / 80; 16 of 2000: 79 / 44
constexpr int kStepRows = 32, kStepRowsFew = 16;

int launch_pages_chunk(const PgParams& p, const PaArgs& a, int dim, uint32_t flags, cudaStream_t s);

}  // namespace less
