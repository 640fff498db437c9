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
//     over blocks (a counter that the last one resets; the order of the sum is fixed).
//   - A tile lies in memory in the order of the mma operand fragments (pages.cuh), so a lane copies (cp.async) and
//     reads back the very bytes it needs: no barrier, no transposition, no bank conflicts.
//   - Scores are computed transposed (m16n8k16: 16 tokens x 16 dimensions of K times 8 query rows): eight rows fill an
//     instruction, and the codes, converted to fp16 exactly, are never scaled - the magnitude of a key block
//     multiplies its scores, that of a value block its probabilities.
//   - The running maximum of a row is only a reference: it is replaced, and the sums rescaled, when a score exceeds it
//     by 2^8, which one vote per block finds; a block costs no shuffles otherwise.
// Roundings: bf16 queries become fp16 after division by a power of two of their row (11 bits are enough for 8; what
// lies 2^-14 below the row's largest loses bits, 2^-25 of the largest at most).  Probabilities times magnitude go
// into the second product as fp16 high part plus fp16 rest (22 bits), relative to a power of two of the largest value
// magnitude so far, so the sums are as good as fp32 wherever magnitudes of a context lie within 2^14 of each other.
// The output is rounded once.
#include <atomic>
#include <type_traits>

#include "less_internal.cuh"
#include "pages_attn.cuh"

namespace less {

constexpr int PS_WARPS = 8, PS_THREADS = PS_WARPS * 32;
constexpr int PS_STAGES = 3;
constexpr int PS_MIN_BLOCKS = 2;               // blocks a warp takes at least: below that, merging costs more
constexpr int PS_SLOT_FLOATS = 2112;           // rows x (D + 2) floats: 16 x 130 or 32 x 66

// 128 registers a thread hold the sums and queries of eight rows; more rows take what one block per SM leaves
__host__ __device__ constexpr int ps_blocks_per_sm(int NT) { return NT == 1 ? 2 : 1; }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
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

__device__ __forceinline__ void store4(__half* dst, float4 f) {
  __half2 h[2] = {__floats2half2_rn(f.x, f.y), __floats2half2_rn(f.z, f.w)};
  *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<uint2*>(h);
}
__device__ __forceinline__ void store4(__nv_bfloat16* dst, float4 f) {
  __nv_bfloat162 h[2] = {__floats2bfloat162_rn(f.x, f.y), __floats2bfloat162_rn(f.z, f.w)};
  *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<uint2*>(h);
}

// One item: rows [row0, row0 + valid) of a (sequence, layer, head)'s tokens x group rows.
struct Item {
  int64_t begin;                // first block in the list of all blocks
  int blocks;
  int valid;                    // rows of this item
  int h, row0, tok_row, lj;
};

struct PsShared {
  int64_t pre[PS_THREADS + 1];  // blocks of the entries before a thread's
  Item part[PS_WARPS][2];       // the item that a warp's slot 0 / 1 holds a part of
  int has[PS_WARPS][2];
  Item fin[2];                  // items that this block merges over all blocks
  int fin_on[2];
};

// address of an item's row: rows are (token, query head of the group)
__device__ __forceinline__ int64_t row_offset(const PgParams& p, const PaArgs& a, int D, const Item& it, int r) {
  const int rr = it.row0 + r, tok = rr / p.group, hd = rr - tok * p.group;
  return ((int64_t)(it.tok_row + tok) * a.nl + it.lj) * ((int64_t)p.heads * p.group * D) +
         ((int64_t)it.h * p.group + hd) * D;
}

template <typename T, int D, int NT, bool E4M3>
__global__ void __launch_bounds__(PS_THREADS, ps_blocks_per_sm(NT)) pages_step_kernel(PgParams p, PaArgs a) {
  constexpr int R = 8 * NT, MT = D / 16, KS = D / 16;
  constexpr int TILE = 16 * D, CH = TILE / 512;           // bytes of a tile; 16-byte pieces per lane
  constexpr int SLOT = R * (D + 2);
  static_assert(SLOT <= PS_SLOT_FLOATS, "slot");
  extern __shared__ __align__(16) unsigned char ps_ring[];
  __shared__ PsShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;

  // ---- the list of blocks: a thread counts the entries of a stretch of its own, one scan orders them ----
  const int per_thread = pg_ceil(a.n, PS_THREADS);
  auto entry_units = [&](const PgEntry& e, Blocks& b, int& tiles) -> int64_t {
    const int64_t nr = (int64_t)e.count * p.group;
    if (nr == 0 || nr > a.max_rows) return 0;
    b = visible_blocks(a, e.len, e.count);
    tiles = (int)((nr + R - 1) / R);
    return (int64_t)max(1, b.count()) * tiles * a.nl * p.heads;
  };
  {
    int64_t mine = 0;
    for (int i = tid * per_thread; i < min(a.n, (tid + 1) * per_thread); ++i) {
      Blocks b;
      int tiles;
      mine += entry_units(pg_entry(p, a.seqs, a.starts, a.rows, i), b, tiles);
    }
    int64_t x = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += y;
    }
    __shared__ int64_t sums[PS_WARPS];
    if (lane == 31) sums[warp] = x;
    if (tid < 2 * PS_WARPS) sh.has[tid >> 1][tid & 1] = 0;
    if (tid < 2) sh.fin_on[tid] = 0;
    __syncthreads();
    for (int w = 0; w < warp; ++w) x += sums[w];
    sh.pre[tid + 1] = x;
    if (tid == 0) sh.pre[0] = 0;
    __syncthreads();
  }
  const int64_t total = sh.pre[PS_THREADS];
  const int64_t workers = (int64_t)gridDim.x * PS_WARPS;
  const int64_t per_warp = max((total + workers - 1) / workers, (int64_t)PS_MIN_BLOCKS);
  const int64_t cta_begin = (int64_t)blockIdx.x * PS_WARPS * per_warp;
  if (cta_begin >= total) return;
  const int64_t cta_end = min(total, cta_begin + PS_WARPS * per_warp);
  int64_t u = min(total, cta_begin + warp * per_warp);
  const int64_t ue = min(total, u + per_warp);

  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ps_ring) + warp * (PS_STAGES * 2 * TILE) + lane * 16;
  const unsigned char* ring_g = ps_ring + warp * (PS_STAGES * 2 * TILE) + lane * 16;
  float* slots = p.partial + (size_t)(blockIdx.x * (2 * PS_WARPS + 2)) * PS_SLOT_FLOATS;

  // ---- where this warp starts ----
  int ei = 0, index = 0, bo = 0;            // entry, item of the entry, block of the item
  int64_t entry_begin = 0;
  PgEntry e = {};
  Blocks vb = {};
  int tiles = 1, items = 0;
  if (u < ue) {
    int lo = 0, hi = PS_THREADS - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sh.pre[mid] <= u) lo = mid; else hi = mid - 1;
    }
    ei = lo * per_thread;
    entry_begin = sh.pre[lo];
    for (; ei < a.n; ++ei) {
      e = pg_entry(p, a.seqs, a.starts, a.rows, ei);
      const int64_t nu = entry_units(e, vb, tiles);
      if (u < entry_begin + nu) break;
      entry_begin += nu;
    }
    if (ei >= a.n) u = ue;                  // cannot be, unless the lengths changed under the call
    items = tiles * a.nl * p.heads;
    const int blocks = max(1, vb.count());
    index = (int)((u - entry_begin) / blocks);
    bo = (int)((u - entry_begin) - (int64_t)index * blocks);
  }

  while (u < ue) {
    // ---- the item ----
    const int blocks = max(1, vb.count());
    Item it;
    it.begin = entry_begin + (int64_t)index * blocks;
    it.blocks = blocks;
    it.row0 = (index % tiles) * R;
    it.h = (index / tiles) % p.heads;
    it.lj = index / tiles / p.heads;
    it.tok_row = e.row0;
    it.valid = min(R, e.count * p.group - it.row0);
    const int first = bo, last = (int)min((int64_t)blocks, bo + (ue - u));
    const int layer = a.layer0 + it.lj;

    // ---- its queries: operand fragments, the score factor and the position of the rows of this lane ----
    uint32_t qf[NT][D / 8];
    float crow[NT][2];
    int pos[NT][2];
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
        for (int i = 0; i < D / 32; ++i) w[i] = __ldg(reinterpret_cast<const uint4*>(src) + i);
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
        pos[nt][c] = rc < it.valid ? e.len - e.count + (it.row0 + rc) / p.group : -1;
      }
    }
    const int first_pos = e.len - e.count + it.row0 / p.group, last_pos = e.len - e.count + (it.row0 + it.valid - 1) / p.group;
    const bool all_rows = it.valid == R;

    float o[NT][MT][4], m[NT][2], l[NT][2];
    float vref = 0x1p-126f, ivref = 0x1p126f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[nt][mt][i] = 0.f;
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
    }

    // lane i knows page and magnitudes of block `batch + i` of the item
    int page_l = -1;
    float ak_l = 0.f, av_l = 0.f;
    auto lookup = [&](int batch) {
      page_l = -1;
      if (batch + lane < last && vb.count() > 0) {
        const int tok = vb.at(batch + lane) * kPageBlock;
        page_l = pg_page(p, e.seq, tok >> p.pt_shift);
        if (page_l >= 0) {
          const float* mg = p.amax + pg_mag(p, layer, page_l, it.h) + (tok & (p.pt - 1)) / kPageBlock;
          ak_l = __ldg(mg);
          av_l = __ldg(mg + p.pt / kPageBlock);
        }
      }
    };
    auto fetch = [&](int b, int batch, int stage) {
      const int page = __shfl_sync(0xffffffffu, page_l, (b - batch) & 31);
      if (b < last && page >= 0) {
        const int inner = ((vb.at(b) * kPageBlock) & (p.pt - 1)) / kPageBlock;
        const uint8_t* k = p.codes + pg_slab(p, D, layer, page, it.h) + (size_t)inner * TILE + lane * 16;
        const uint8_t* v = k + (size_t)p.pt * D;
        const uint32_t dst = ring + stage * (2 * TILE);
#pragma unroll
        for (int i = 0; i < CH; ++i) cp_async16(dst + i * 512, k + i * 512);
#pragma unroll
        for (int i = 0; i < CH; ++i) cp_async16(dst + TILE + i * 512, v + i * 512);
      }
      cp_async_commit();
    };

    int stage = 0;
    for (int batch = first; batch < last; batch += 32) {
      lookup(batch);
      const int stop = min(last, batch + 32);
      // the ring restarts with every batch of 32 blocks
      for (int s = 0; s < PS_STAGES - 1; ++s) fetch(batch + s < stop ? batch + s : last, batch, (stage + s) % PS_STAGES);
      for (int b = batch; b < stop; ++b) {
        const int ahead = b + PS_STAGES - 1;
        fetch(ahead < stop ? ahead : last, batch, (stage + PS_STAGES - 1) % PS_STAGES);
        cp_async_wait<PS_STAGES - 1>();
        const int page = __shfl_sync(0xffffffffu, page_l, b - batch);
        const float ak = __shfl_sync(0xffffffffu, ak_l, b - batch), av = __shfl_sync(0xffffffffu, av_l, b - batch);
        const unsigned char* tile = ring_g + stage * (2 * TILE);
        stage = stage + 1 == PS_STAGES ? 0 : stage + 1;
        if (page < 0) continue;                                    // trimmed
        const int j0 = vb.at(b) * kPageBlock;

        // ---- scores: 16 tokens x 8 NT rows ----
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
        for (int half = 0; half < D / 64; ++half) {
          const uint4 k0 = *reinterpret_cast<const uint4*>(tile + half * 512);
          const uint4 k1 = *reinterpret_cast<const uint4*>(tile + (D / 64 + half) * 512);
          const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t a0, a1, a2, a3;
            pg_unpack4<E4M3>(w0[w], a0, a2);
            pg_unpack4<E4M3>(w1[w], a1, a3);
            const int ks = half * 4 + w;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma16816(s[nt], a0, a1, a2, a3, qf[nt][2 * ks], qf[nt][2 * ks + 1]);
          }
        }
        bool up = false;
        const bool whole = all_rows && j0 + kPageBlock - 1 <= first_pos &&
                           (!a.window || j0 > last_pos - a.window || j0 + kPageBlock <= a.sinks);
        // this lane's tokens: accumulator rows g and g + 8
        const int ja = j0 + 4 * (g >> 1) + (g & 1), jb = ja + 2;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int i = 0; i < 4; ++i) s[nt][i] *= ak * crow[nt][i & 1];
          if (!whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int j = i < 2 ? ja : jb, at = pos[nt][i & 1];
              if (j > at || (a.window && j <= at - a.window && j >= a.sinks)) s[nt][i] = -INFINITY;
            }
          }
          up |= fmaxf(s[nt][0], s[nt][2]) > m[nt][0] + 8.f || fmaxf(s[nt][1], s[nt][3]) > m[nt][1] + 8.f;
        }
        if (__any_sync(0xffffffffu, up)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float x = fmaxf(s[nt][c], s[nt][2 + c]);
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
              x = fmaxf(x, m[nt][c]);
              const float f = x == m[nt][c] ? 1.f : pa_ex2(m[nt][c] - x);
              m[nt][c] = x;
              l[nt][c] *= f;
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                o[nt][mt][c] *= f;
                o[nt][mt][2 + c] *= f;
              }
            }
        }
        if (av > 16.f * vref) {
          const float now = __uint_as_float((__float_as_uint(av) & 0x7f800000u) + 0x00800000u);
          ivref = __uint_as_float(0x7f000000u - __float_as_uint(now));
          const float f = vref * ivref;
          vref = now;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[nt][mt][i] *= f;
        }
        // ---- probabilities, times the value magnitude: second operand of the product with the values ----
        const float r = av * ivref;
        uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float mm = m[nt][i & 1];
            x[i] = pa_ex2(s[nt][i] - (mm == -INFINITY ? 0.f : mm));
          }
          l[nt][0] += x[0] + x[2];
          l[nt][1] += x[1] + x[3];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float y0 = x[2 * i] * r, y1 = x[2 * i + 1] * r;
            const __half2 hi = __floats2half2_rn(y0, y1);
            const float2 back = __half22float2(hi);
            ph[nt][i] = movmatrix(*reinterpret_cast<const uint32_t*>(&hi));
            pl[nt][i] = movmatrix(pack2(y0 - back.x, y1 - back.y));
          }
        }
        // tokens behind the end may hold any byte; a NaN code would survive its zero probability
        uint32_t keep = 0xffffffffu;
        if (E4M3 && j0 + kPageBlock > e.len) {
          const int left = e.len - (j0 + 4 * t);
          keep = left <= 0 ? 0u : (left >= 4 ? keep : keep >> (8 * (4 - left)));
        }
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          const uint4 v4 = *reinterpret_cast<const uint4*>(tile + TILE + i * 512);
          const uint32_t w[4] = {v4.x & keep, v4.y & keep, v4.z & keep, v4.w & keep};
#pragma unroll
          for (int dd = 0; dd < 4; dd += 2) {
            uint32_t a0, a1, a2, a3;
            pg_unpack4<E4M3>(w[dd], a0, a2);
            pg_unpack4<E4M3>(w[dd + 1], a1, a3);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma16816(o[nt][2 * i + dd / 2], a0, a1, a2, a3, ph[nt][0], ph[nt][1]);
              mma16816(o[nt][2 * i + dd / 2], a0, a1, a2, a3, pl[nt][0], pl[nt][1]);
            }
          }
        }
      }
      cp_async_wait<0>();
    }

    // ---- the item's rows, or a part of them ----
    const bool complete = first == 0 && last == blocks;
    const int which = first == 0 ? 1 : 0;
    float* slot = slots + (size_t)(warp * 2 + which) * PS_SLOT_FLOATS;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float sum = l[nt][c];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const int rc = nt * 8 + 2 * t + c;
        if (rc >= it.valid) continue;
        const float inv = sum > 0.f ? 1.f / sum : 0.f, unit = vref / pg_top<E4M3>();
        float f[D / 8];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          f[2 * mt] = o[nt][mt][c] * inv * unit;
          f[2 * mt + 1] = o[nt][mt][2 + c] * inv * unit;
        }
        if (sum != sum) {                                    // a query that is not finite
#pragma unroll
          for (int i = 0; i < D / 8; ++i) f[i] = sum;
        }
        if (complete) {
          T* dst = reinterpret_cast<T*>(a.out) + row_offset(p, a, D, it, rc) + g * (D / 8);
#pragma unroll
          for (int i = 0; i < D / 8; i += 8) store8<T>(dst + i, f + i);
        } else {
          float* dst = slot + rc * D + g * (D / 8);
#pragma unroll
          for (int i = 0; i < D / 8; i += 4) *reinterpret_cast<float4*>(dst + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
          if (g == 0) {
            slot[R * D + 2 * rc] = m[nt][c];
            slot[R * D + 2 * rc + 1] = sum;
          }
        }
      }
    if (!complete && lane == 0) {
      sh.part[warp][which] = it;
      sh.has[warp][which] = 1;
    }

    // ---- next ----
    u += last - first;
    bo = 0;
    if (++index == items && u < ue) {
      index = 0;
      entry_begin += (int64_t)items * blocks;
      do {
        if (++ei >= a.n) break;
        e = pg_entry(p, a.seqs, a.starts, a.rows, ei);
      } while (entry_units(e, vb, tiles) == 0);
      if (ei >= a.n) break;                 // as above
      items = tiles * a.nl * p.heads;
    }
  }
  __syncthreads();

  // ---- merge inside the block: the warp that holds an item's first part in this block collects the others ----
  auto merge_rows = [&](const Item& it, auto slot_of, int parts, int r, float4& f, float& mm, float& ll) {
    // one row, a warp: lanes own four dimensions each (two halves of the warp alternate when D is 64)
    const int c4 = (lane % (D / 4)) * 4;
    mm = -INFINITY;
    for (int i = lane; i < parts; i += 32) mm = fmaxf(mm, __ldcg(slot_of(i) + R * D + 2 * r));
#pragma unroll
    for (int d = 16; d; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
    f = make_float4(0.f, 0.f, 0.f, 0.f);
    ll = 0.f;
#pragma unroll 4
    for (int i = 0; i < parts; ++i) {
      const float* s = slot_of(i);
      const float pm = __ldcg(s + R * D + 2 * r), pl = __ldcg(s + R * D + 2 * r + 1);
      const float4 v = __ldcg(reinterpret_cast<const float4*>(s + r * D + c4));
      const float w = pl == 0.f ? 0.f : pl * pa_ex2(pm - mm);
      ll += w;
      f.x = fmaf(w, v.x, f.x);
      f.y = fmaf(w, v.y, f.y);
      f.z = fmaf(w, v.z, f.z);
      f.w = fmaf(w, v.w, f.w);
    }
    const float inv = ll == 0.f ? 0.f : 1.f / ll;
    f = make_float4(f.x * inv, f.y * inv, f.z * inv, f.w * inv);
  };
  const int64_t per_cta = PS_WARPS * per_warp;
  for (int which = 0; which < 2; ++which) {
    if (!sh.has[warp][which] || (which == 0 && warp != 0)) continue;
    const Item it = sh.part[warp][which];
    const int64_t end = it.begin + it.blocks;
    const int wl = (int)((min(end, cta_end) - 1 - cta_begin) / per_warp);
    const bool inside = it.begin >= cta_begin && end <= cta_end;
    float* cta_slot = slots + (size_t)(2 * PS_WARPS + which) * PS_SLOT_FLOATS;
    const float* base = slots;
    const int w0 = warp, wh = which;
    auto slot_of = [=](int i) { return base + (size_t)((w0 + i) * 2 + (i == 0 ? wh : 0)) * PS_SLOT_FLOATS; };
    for (int r = 0; r < it.valid; ++r) {
      float4 f;
      float mm, ll;
      merge_rows(it, slot_of, wl - warp + 1, r, f, mm, ll);
      if (lane < D / 4) {
        if (inside) {
          store4(reinterpret_cast<T*>(a.out) + row_offset(p, a, D, it, r) + lane * 4, f);
        } else {
          *reinterpret_cast<float4*>(cta_slot + r * D + lane * 4) = f;
          if (lane == 0) {
            cta_slot[R * D + 2 * r] = mm;
            cta_slot[R * D + 2 * r + 1] = ll;
          }
        }
      }
    }
    if (!inside) {
      __threadfence();
      __syncwarp();
      if (lane == 0) {
        const int c0 = (int)(it.begin / per_cta), c1 = (int)((end - 1) / per_cta);
        if (atomicAdd(p.counters + c0, 1) == c1 - c0) {
          p.counters[c0] = 0;
          __threadfence();
          sh.fin[which] = it;
          sh.fin_on[which] = 1;
        }
      }
    }
  }
  __syncthreads();

  // ---- merge over the blocks: the last one to arrive does it, all its warps, a row each ----
  for (int which = 0; which < 2; ++which) {
    if (!sh.fin_on[which]) continue;
    const Item it = sh.fin[which];
    const int c0 = (int)(it.begin / per_cta), c1 = (int)((it.begin + it.blocks - 1) / per_cta);
    const float* base = p.partial;
    auto slot_of = [=](int i) {
      return base + ((size_t)(c0 + i) * (2 * PS_WARPS + 2) + 2 * PS_WARPS + (i == 0 ? 1 : 0)) * PS_SLOT_FLOATS;
    };
    for (int r = warp; r < it.valid; r += PS_WARPS) {
      float4 f;
      float mm, ll;
      merge_rows(it, slot_of, c1 - c0 + 1, r, f, mm, ll);
      if (lane < D / 4) store4(reinterpret_cast<T*>(a.out) + row_offset(p, a, D, it, r) + lane * 4, f);
    }
  }
}

template <typename T, int D, int NT, bool E4M3>
static int launch_step(const PgParams& p, const PaArgs& a, cudaStream_t s) {
  constexpr size_t smem = (size_t)PS_WARPS * PS_STAGES * 2 * 16 * D;
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return fail_cuda("cudaGetDevice");
  if (dev >= 64 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
    if (cudaFuncSetAttribute(pages_step_kernel<T, D, NT, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)smem) != cudaSuccess)
      return fail_cuda("shared memory opt-in of pages_step_kernel");
    if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  constexpr size_t block_bytes = (size_t)(2 * PS_WARPS + 2) * PS_SLOT_FLOATS * 4;
  int grid = ps_blocks_per_sm(NT) * pg_sms();
  const int most = (int)(LESS_PAGES_PARTIAL_BYTES / block_bytes);
  if (grid > most) grid = most;
  if (grid > kPgCounters) grid = kPgCounters;
  pages_step_kernel<T, D, NT, E4M3><<<grid, PS_THREADS, smem, s>>>(p, a);
  return check_launch("pages_step_kernel");
}

template <typename T, bool E4M3>
static int launch_step_dim(const PgParams& p, const PaArgs& a, int dim, int rows, cudaStream_t s) {
  if (dim == 128) return rows > 8 ? launch_step<T, 128, 2, E4M3>(p, a, s) : launch_step<T, 128, 1, E4M3>(p, a, s);
  if (rows > 16) return launch_step<T, 64, 4, E4M3>(p, a, s);
  return rows > 8 ? launch_step<T, 64, 2, E4M3>(p, a, s) : launch_step<T, 64, 1, E4M3>(p, a, s);
}

}  // namespace less

using namespace less;

extern "C" int less_pages_attention(const less_pages* d, int32_t layer_begin, int32_t layer_count, int32_t n,
                                    const int32_t* seqs, const int32_t* starts, int32_t rows, int32_t max_new,
                                    const void* q, int64_t q_stride, int32_t window, int32_t sinks, float scale,
                                    void* out, void* stream) {
  PgParams p;
  int rc = pg_view(d, &p);
  if (rc != LESS_OK) return rc;
  if (layer_begin < 0 || layer_count < 1 || layer_begin > d->layers - layer_count) return LESS_ERR_BAD_LAYER_RANGE;
  if (n < 0 || n > (1 << 24) || rows < 0 || (!starts && rows != n) || max_new < 1) return LESS_ERR_INVALID_CONFIG;
  if (window < 0 || sinks < 0 || !(scale > 0.f) || scale > 3e38f) return LESS_ERR_INVALID_CONFIG;
  if ((int64_t)rows * d->group > 0x7fffffff) return LESS_ERR_INVALID_CONFIG;
  if (n == 0 || rows == 0) return LESS_OK;
  if (!seqs || !q || !out) return LESS_ERR_NULL_POINTER;
  if (((uintptr_t)seqs | (uintptr_t)starts) & 3) return LESS_ERR_MISALIGNED;
  if (q_stride < (int64_t)layer_count * d->heads * d->group * d->head_dim) return LESS_ERR_INVALID_CONFIG;
  if ((((uintptr_t)q | (uintptr_t)out) & 15) || (q_stride & 7)) return LESS_ERR_MISALIGNED;
  // no position reaches 2^30
  PaArgs a = {q, out, q_stride, seqs, starts, n, rows, layer_begin, layer_count, 0x7fffffff,
              window > (1 << 30) ? 0 : window, sinks > (1 << 30) ? 1 << 30 : sinks, scale};
  if (!starts) max_new = 1;
  const int64_t most = (int64_t)max_new * d->group;
  int r = most > 0x7fffffff ? 0x7fffffff : (int)most;
  cudaStream_t s = (cudaStream_t)stream;
  if (r > kStepRows) {
    a.max_rows = kStepRows;
    rc = launch_pages_chunk(p, a, d->head_dim, d->flags, s);
    if (rc != LESS_OK || !starts || d->group > kStepRows) return rc;   // without starts all entries are alike
    r = kStepRows;
  }
  if (d->flags & LESS_PAGES_BF16)
    return (d->flags & LESS_PAGES_E4M3) ? launch_step_dim<__nv_bfloat16, true>(p, a, d->head_dim, r, s)
                                        : launch_step_dim<__nv_bfloat16, false>(p, a, d->head_dim, r, s);
  return (d->flags & LESS_PAGES_E4M3) ? launch_step_dim<__half, true>(p, a, d->head_dim, r, s)
                                      : launch_step_dim<__half, false>(p, a, d->head_dim, r, s);
}
