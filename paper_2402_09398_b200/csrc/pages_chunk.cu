// Attention of many new tokens over the paged 8-bit cache (the chunk kernel): the same result as the step kernel
// (pages_attn.cu) where a sequence brings enough rows - tokens x query heads of a KV head - to fill tensor-core tiles.
//
// 4 D flops and one exponential per visible (query, key) pair; codes are read once per 256 rows, mostly from L2.  One CTA
// = 256 rows of one (sequence, layer, KV head) as two tiles of 128 (a tensor-memory lane per row), late rows first; key
// tiles of 64 tokens, four stages, 14 warps:
//   warps 8 - 11   codes -> fp16 operand tiles in shared memory, two warps per key tile, pairs in turn.  A stored tile is
//                  read with coalesced 16-byte loads straight into registers (the next tile's while this one is
//                  converted), so there is no staging; both operands are written K-major with the 128-byte swizzle,
//                  free of bank conflicts: the keys of a tile are ordered (token groups of 4, alternating between two
//                  stored tiles) such that the four tokens that a stored value word holds, of two tiles, are one
//                  16-byte piece of V^T.
//   warp 12        S = Q K^T                tcgen05, 128 x 64, fp32 in tensor memory, two buffers per row tile
//   warps 0 - 7    softmax, a thread per row: P over S as the A operand of
//   warp 13        O += P V                 tcgen05, A from tensor memory, fp32 accumulator in tensor memory
// While a row tile is in softmax, the tensor cores work on its other buffer and on the other row tile.
// Codes are exact in fp16 and are never scaled.  The magnitude a_k of a key block is part of the factor that turns a
// score into the exponent, and that of a value block, as log2 a_v, part of the exponent's offset:
//   P = 2^(s a_k c + log2 a_v - M)            sum of the probabilities: sum over blocks of (sum P) / a_v
// M is a reference of a row that follows its keys up and down (pages_attn.cuh): scores are exponentiated against the M at
// hand in one pass, and only if the largest exponent lies outside the range around it - as a rule in the first tile alone -
// O and the sums are rescaled and the pass repeated.
// Roundings: P is rounded once to fp16, 2^-11 of each with independent signs or, where it is below 2^-14, 2^-25, which is at
// most 2^-18 of the largest of the key tile; queries as in the step kernel, the output once.
//
// Measured: five sequences of 700 to 8000 tokens, 1 to 2048 of them new, 8 KV heads x 4 queries of D 128: 613 to 650 us,
// 800 to 850 TFLOP/s, half of the matrix rate; 8192 new tokens, 32 heads, window 1024: 265 us (129 GFLOP: 487 TFLOP/s,
// 11 of a CTA's 38 us are its beginning and end).  A key tile of 256 rows takes some 2200 cycles: 1024 of the exponential
// unit, 1250 or more of the tensor cores, and chains of waits between the roles; none is busy much more than half the time.
// Measured and slower (2048 new tokens at 8192, 8 x 4 heads, 307 us then): key tiles of 128 with one score buffer
// 354, with halves 363, with 16 softmax warps 338; 64 with 16 softmax warps 356; codes staged by bulk copies 334;
// conversion by separate warps for K and V 380.
#include <atomic>
#include <type_traits>

#include "less_internal.cuh"
#include "pages_attn.cuh"
#include "tc_common.cuh"

namespace less {

constexpr int PC_ROWS = 128, PC_KEYS = 64;
constexpr int PC_TILES = PC_KEYS / kPageBlock;            // stored tiles of a key tile
constexpr int PC_SOFT_WARPS = 8, PC_DEQ_WARPS = 4;
constexpr int PC_THREADS = (PC_SOFT_WARPS + PC_DEQ_WARPS + 2) * 32;
constexpr int PC_STAGES = 4, PC_META = 8;
constexpr float PC_WIDE = 64.f;                           // log2 of magnitudes that far apart need care (see the softmax)
constexpr int PC_POLY = 1;                                // of eight pairs of exponentials, those on the FMA pipe (see ex2_poly)

struct __align__(16) PcMeta {                                           // of the stored tiles of a key tile
  float k1[PC_TILES];                                     // a_k / top
  float lav[PC_TILES], iav[PC_TILES];                     // log2 a_v, 1 / a_v
  int j0[PC_TILES];                                       // position of the first token, 2^30 = no tile
  uint32_t part[PC_TILES];                                // bit x: row tile x does not see all of it; [0] bit 2: PC_WIDE
};

struct PcShared {
  uint64_t q_full, k_full[PC_STAGES], k_empty[PC_STAGES], v_full[PC_STAGES], v_empty[PC_STAGES];
  uint64_t s_full[2][2], p_full[2][2], pv_done[2][2];     // [row tile][buffer]: key tiles alternate
  PcMeta meta[PC_META];
  float lowest[2 * PC_ROWS];                              // how far down the references of the rows may go
  uint32_t tmem_base;
  int abort;
};

// 2^y for two values on the FMA pipe, y >= -126 (smaller counts as that): y = n + f with n the nearest integer, 2^f by a
// polynomial of degree 4 (least maximum of the relative error on [-1/2, 1/2]: 2.6e-6, 2^-18.6), n added to its exponent.
// The exponential unit gives one result in eight cycles per warp, 16 per SM and cycle: of a key tile's exponentials it
// takes as many cycles as the tensor cores of the products, so PC_POLY of every eight pairs are computed here (8 KV heads x 4,
// 2048 new tokens at 8192: none 280 us, one 277, two 304, four 342: instruction slots are scarce too).
__device__ __forceinline__ void ex2_poly(float y0, float y1, float& p0, float& p1) {
  const uint64_t y = f32x2_pack(fmaxf(y0, -126.f), fmaxf(y1, -126.f)), magic = f32x2_pack(12582912.f, 12582912.f);
  const uint64_t t = f32x2_add(y, magic);                // n in the low bits
  const uint64_t f = f32x2_fma(f32x2_add(t, f32x2_pack(-12582912.f, -12582912.f)), f32x2_pack(-1.f, -1.f), y);
  uint64_t g = f32x2_pack(0.009570101276f, 0.009570101276f);
  g = f32x2_fma(g, f, f32x2_pack(0.055917859077f, 0.055917859077f));
  g = f32x2_fma(g, f, f32x2_pack(0.240247443318f, 0.240247443318f));
  g = f32x2_fma(g, f, f32x2_pack(0.693121790886f, 0.693121790886f));
  g = f32x2_fma(g, f, f32x2_pack(0.999999284744f, 0.999999284744f));
  float t0, t1;
  f32x2_unpack(t, t0, t1);
  f32x2_unpack(g, p0, p1);
  p0 = __uint_as_float(__float_as_uint(p0) + (__float_as_uint(t0) << 23));
  p1 = __uint_as_float(__float_as_uint(p1) + (__float_as_uint(t1) << 23));
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      :
      : "r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
        "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
        "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}

// The issuing warps stay converged and only the instruction itself is predicated on one elected lane: operands then
// live in uniform registers.  Issued from a divergent branch, each MMA first moves its operands there one by one - 108
// against 77 cycles per MMA measured here (no softmax, no conversion), 1.4 x on the whole.
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t on;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(on));
  return on;
}
// a descriptor moved by `off` 16-byte units (addresses stay below 2^18: the low word does not carry over)
__device__ __forceinline__ uint64_t desc_at(uint64_t d, uint32_t off) {
  return (d & 0xffffffff00000000ull) | (uint32_t)((uint32_t)d + off);
}
__device__ __forceinline__ void mma_ss_if(uint32_t on, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                          uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}
__device__ __forceinline__ void mma_ts_if(uint32_t on, uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                          uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(on)
      : "memory");
}
__device__ __forceinline__ void mma_commit_if(uint32_t on, uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)),
      "r"(on)
      : "memory");
}

// Slots of the grid: entry i owns slots [starts[i] G / 256 + i, starts[i + 1] G / 256 + i + 1) - at least as many as it
// has pairs of row tiles
__device__ __forceinline__ int64_t pc_slot(const PgParams& p, const PaArgs& a, int i) {
  const int row = a.starts ? min(max(__ldg(a.starts + i), 0), a.rows) : i;
  return (int64_t)row * p.group / (2 * PC_ROWS) + i;
}

constexpr int PC_SPLIT_TILES = 4;                         // key tiles of a split CTA at least

// where the CTA of (slot, head, split) leaves its part: rows x D values, then (reference, sum) of the rows
__device__ __forceinline__ size_t pc_part(int64_t slot, int heads, int head, int splits, int split, int D) {
  return ((size_t)(slot * heads + head) * splits + split) * ((size_t)2 * PC_ROWS * (D + 2));
}

// visibility of the 32 columns of a stored-tile pair, bit 16 e + r = token r of tile e
__device__ __forceinline__ uint32_t pc_mask16(int j0, int pos, int window, int sinks) {
  const int hi = min(max(pos + 1 - j0, 0), 16);
  uint32_t m = (1u << hi) - 1;                            // j <= pos
  if (window) {
    const int lo = min(max(pos - window + 1 - j0, 0), 16), sk = min(max(sinks - j0, 0), 16);
    m &= ~((1u << lo) - 1) | ((1u << sk) - 1);
  }
  return m & 0xffffu;
}

template <typename T, int D, bool E4M3>
__global__ void __launch_bounds__(PC_THREADS, 1) pages_chunk_kernel(PgParams p, PaArgs a, int splits) {
  constexpr int QT = PC_ROWS * D * 2;                     // bytes of a Q tile
  constexpr int KT = PC_KEYS * D * 2;                     // of a K or V tile
  extern __shared__ __align__(1024) unsigned char pc_smem[];
  unsigned char* qres = pc_smem;                          // [2 row tiles][D / 64][128 rows][128 B]
  unsigned char* kring = qres + 2 * QT;                   // [stages][D / 64][64 keys][128 B]
  unsigned char* vring = kring + PC_STAGES * KT;          // [stages][D dims][128 B]
  PcShared* sh = reinterpret_cast<PcShared*>(vring + PC_STAGES * KT);
  if (smem_misaligned(pc_smem, p.status, 120)) return;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pg_wait();
  if (blockIdx.x == gridDim.x - 1) {                      // one CTA more than there are slots
    if (blockIdx.y == 0) pg_check_starts(p, a.starts, a.n);
    return;
  }
  // ---- the item: late rows, which see most, first ----
  const int heads = a.nl * p.heads, lh = (int)(blockIdx.x % heads);         // layer and head
  const int64_t slot = (gridDim.x - 1) / heads - 1 - blockIdx.x / heads;
  int lo = 0, hi = a.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pc_slot(p, a, mid) <= slot) lo = mid; else hi = mid - 1;
  }
  const PgEntry e = pg_entry(p, a.seqs, a.starts, a.rows, lo);
  const int64_t rows = (int64_t)e.count * p.group;
  const int64_t row0 = (slot - pc_slot(p, a, lo)) * (2 * PC_ROWS);
  // the step kernel's, or a slot before the first entry's (its rows need not start at 0), or no rows left
  if (rows <= a.max_rows || row0 < 0 || row0 >= rows) return;
  const int valid = (int)min(rows - row0, (int64_t)2 * PC_ROWS), nx = valid > PC_ROWS ? 2 : 1;
  const int lj = lh / p.heads, h = lh - lj * p.heads, layer = a.layer0 + lj;
  const int base = e.len - e.count;                       // position of the entry's first token
  const int tok0 = (int)(row0 / p.group), tok1 = (int)((row0 + valid - 1) / p.group);
  const Blocks vb = visible_blocks(a, base + tok1 + 1, tok1 - tok0 + 1);
  const int units = base + tok1 < 0 ? 0 : vb.count();
  // with few items the key tiles are dealt out to `splits` CTAs (blockIdx.y), whose results are joined by a second kernel
  const int nk_all = pg_ceil(units, PC_TILES), share = max(pg_ceil(nk_all, splits), splits > 1 ? PC_SPLIT_TILES : 1);
  const int kt0 = min(nk_all, (int)blockIdx.y * share), nk = min(share, nk_all - kt0);
  float* part = p.partial + pc_part(slot, heads, lh, splits, blockIdx.y, D);
  const int64_t head_row = ((int64_t)lj * p.heads + h) * p.group * D;
  T* out = reinterpret_cast<T*>(a.out);

  if (nk == 0) {                                          // nothing to see
    if (splits > 1) {
      for (int i = tid; i < valid; i += PC_THREADS)
        *reinterpret_cast<float2*>(part + (size_t)2 * PC_ROWS * D + 2 * i) = make_float2(-INFINITY, 0.f);
      return;
    }
    for (int i = tid; i < valid * (D / 8); i += PC_THREADS) {
      const int64_t rr = row0 + i / (D / 8);
      const int tok = (int)(rr / p.group), hd = (int)(rr - (int64_t)tok * p.group);
      *reinterpret_cast<uint4*>(out + (int64_t)(e.row0 + tok) * a.nl * p.heads * p.group * D + head_row + hd * D +
                                i % (D / 8) * 8) = make_uint4(0, 0, 0, 0);
    }
    return;
  }

  if (tid == 0) {
    mbar_init(&sh->q_full, 4 * nx);
    for (int s = 0; s < PC_STAGES; ++s) {
      mbar_init(&sh->k_full[s], PC_DEQ_WARPS / 2);
      mbar_init(&sh->k_empty[s], 1);
      mbar_init(&sh->v_full[s], PC_DEQ_WARPS / 2);
      mbar_init(&sh->v_empty[s], 1);
    }
    for (int x = 0; x < 4; ++x) {
      mbar_init(&sh->s_full[x >> 1][x & 1], 2);
      mbar_init(&sh->p_full[x >> 1][x & 1], 4);
      mbar_init(&sh->pv_done[x >> 1][x & 1], 1);
    }
    sh->abort = 0;
    mbar_fence_init();
  }
  if (warp == 12) tmem_alloc(&sh->tmem_base, 512);
  fence_proxy_async_smem();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = sh->tmem_base;
  constexpr uint32_t OCOL = 4 * PC_KEYS;                  // S / P of the two row tiles, two buffers each; accumulators
  volatile int* abortp = &sh->abort;
  int32_t* status = p.status;

  if (warp < PC_SOFT_WARPS) {
    // ---------------- softmax: thread = row ----------------
    const int x = warp >> 2, quad = warp & 3;
    if (x < nx) {
      const int r = x * PC_ROWS + quad * 32 + lane;
      const int64_t rr = row0 + min(r, valid - 1);
      const int tok = (int)(rr / p.group), hd = (int)(rr - (int64_t)tok * p.group);
      const int pos = base + tok;
      // the row's query, as fp16, into the operand tile
      float crow = a.scale * 1.4426950408889634f;
      {
        const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(a.q) + (int64_t)(e.row0 + tok) * a.q_stride +
                                                          head_row + hd * D);
        unsigned char* dst = qres + x * QT + (r & (PC_ROWS - 1)) * 128;
        float down = 1.f;
        if (!std::is_same<T, __half>::value) {
          float most = 0.f;
#pragma unroll
          for (int c = 0; c < D / 8; ++c) {
            const uint4 w = __ldcg(src + c);
            const __nv_bfloat162* y = reinterpret_cast<const __nv_bfloat162*>(&w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 f = __bfloat1622float2(y[i]);
              most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
          }
          const int ex = min(max((int)(__float_as_uint(most) >> 23), 1), 253);
          crow *= __uint_as_float((uint32_t)ex << 23);
          down = __uint_as_float((uint32_t)(254 - ex) << 23);
        }
#pragma unroll
        for (int c = 0; c < D / 8; ++c) {
          uint4 w = r < valid ? __ldcg(src + c) : make_uint4(0, 0, 0, 0);
          if (!std::is_same<T, __half>::value) {
            const __nv_bfloat162* y = reinterpret_cast<const __nv_bfloat162*>(&w);
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 f = __bfloat1622float2(y[i]);
              u[i] = pack2(f.x * down, f.y * down);
            }
            w = make_uint4(u[0], u[1], u[2], u[3]);
          }
          *reinterpret_cast<uint4*>(dst + (c >> 3) * (QT / (D / 64)) + (((c & 7) ^ (r & 7)) << 4)) = w;
        }
        fence_proxy_async_smem();
        mbar_arrive_warp(&sh->q_full);
      }

      const uint32_t lane_addr = tmem + ((uint32_t)(quad * 32) << 16);
      const uint32_t ocol = lane_addr + OCOL + x * D;
      float M = -INFINITY, l = 0.f;
      for (int kt = 0; kt < nk; ++kt) {
        const int buf = kt & 1;
        const uint32_t scol = lane_addr + (2 * x + buf) * PC_KEYS;
        wait_or_give_up(&sh->s_full[x][buf], (kt >> 1) & 1, abortp, status, 122);
        __syncwarp();                                     // after a give-up all waits return at once: no way out needed
        tc_fence_after_sync();
        const PcMeta& meta = sh->meta[kt % PC_META];
        const uint4 part = *reinterpret_cast<const uint4*>(meta.part);
        const float4 k1 = *reinterpret_cast<const float4*>(meta.k1), lav = *reinterpret_cast<const float4*>(meta.lav),
                     iav = *reinterpret_cast<const float4*>(meta.iav);
        const bool masked = (part.x | part.y | part.z | part.w) >> x & 1;

        uint32_t pk[PC_KEYS / 2];
        float most, add;
        auto pass = [&](auto with_mask, float ref) {
          most = -INFINITY;
          add = 0.f;
#pragma unroll
          for (int c = 0; c < PC_KEYS / 32; ++c) {        // a pair of stored tiles: 4 columns of one, 4 of the other, ...
            uint32_t s[32];
            tmem_ld32(scol + 32 * c, s);
            const float ke = (c ? k1.z : k1.x) * crow, ko = (c ? k1.w : k1.y) * crow;
            const float be = (c ? lav.z : lav.x) - ref, bo = (c ? lav.w : lav.y) - ref;
            uint32_t m = 0xffffffffu;
            if (decltype(with_mask)::value)
              m = pc_mask16(meta.j0[2 * c], pos, a.window, a.sinks) |
                  pc_mask16(meta.j0[2 * c + 1], pos, a.window, a.sinks) << 16;
            const uint64_t k2[2] = {f32x2_pack(ke, ke), f32x2_pack(ko, ko)}, b2[2] = {f32x2_pack(be, be), f32x2_pack(bo, bo)};
            uint64_t sum[2] = {0, 0};
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) {                // columns 2 i, 2 i + 1
              const int ev = (i >> 1) & 1, tokbit = 16 * ev + 4 * (i >> 2) + 2 * (i & 1);
              float y0, y1;
              f32x2_unpack(f32x2_fma(f32x2_pack(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), k2[ev], b2[ev]), y0, y1);
              if (decltype(with_mask)::value) {
                y0 = m >> tokbit & 1 ? y0 : -INFINITY;
                y1 = m >> (tokbit + 1) & 1 ? y1 : -INFINITY;
              }
              most = fmaxf(most, fmaxf(y0, y1));
              float p0, p1;
              if (!decltype(with_mask)::value && i % 8 >= 8 - PC_POLY) {   // nothing is masked here: no zeros are needed
                ex2_poly(y0, y1, p0, p1);
              } else {
                p0 = pa_ex2(y0);
                p1 = pa_ex2(y1);
              }
              sum[ev] = f32x2_add(sum[ev], f32x2_pack(p0, p1));
              pk[16 * c + i] = pack2(p0, p1);
            }
            float e0, e1, o0, o1;
            f32x2_unpack(sum[0], e0, e1);
            f32x2_unpack(sum[1], o0, o1);
            add = fmaf(e0 + e1, c ? iav.z : iav.x, fmaf(o0 + o1, c ? iav.w : iav.y, add));
          }
        };
        for (bool again = false;; again = true) {
          const float ref = M == -INFINITY ? 0.f : M;
          if (masked) {
            pass(std::true_type{}, ref);
            // P / a_v is the probability as long as P does not underflow, which it does beside values 2^126 larger.  In a
            // tile with a block 2^64 below the largest magnitude so far (an all-zero one beside others, as a rule) the
            // probabilities are summed from exponentials without a_v; nearer ones lose less than 2^-62 of the sum each.
            // Only masked tiles look (a bit that the issuing warp sets makes such a tile one): after either kind of pass
            // the same loop took 14 % of the whole, through registers.
            if (part.x & 4) {
              add = 0.f;
#pragma unroll 1
              for (int c = 0; c < PC_KEYS / 8; ++c) {     // four tokens of each tile of a pair
                uint32_t s[8];
                tmem_ld8(scol + 8 * c, s);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                  const int b = 2 * (c >> 2) + (i >> 2);
                  if (pc_mask16(meta.j0[b], pos, a.window, a.sinks) >> (4 * (c & 3) + (i & 3)) & 1)
                    add += pa_ex2(fmaf(__uint_as_float(s[i]), meta.k1[b] * crow, -ref));
                }
              }
            }
          } else {
            pass(std::false_type{}, ref);
          }
          const bool none = M == -INFINITY, up = most > (none ? -INFINITY : kRefMost);
          const bool down = !none && most < kRefLeast && most > -INFINITY;
          if (again || !__any_sync(0xffffffffu, up || down)) break;
          float d = up || down ? most - (up && !none ? kRefUp : kRefNew) : 0.f;   // what the reference moves by
          const float lowest = none ? -INFINITY : sh->lowest[r];
          // down by 40 below the highest, so that O has room, and no further than l has
          if (down) d = fmaxf(d, fmaxf(lowest - M, (float)min(0, (int)(__float_as_uint(l) >> 23) - 127 - 90)));
          if (up) sh->lowest[r] = fmaxf(lowest, ref + d - 40.f);
          if (up || down) {
            M = ref + d;
            d = M - ref;                                  // as it is rounded
          }
          if (none) d = 0.f;
          l = pa_scaled(l, -d);
          const float f = pa_ex2(-d);
          if (kt) {
            wait_or_give_up(&sh->pv_done[x][(kt - 1) & 1], ((kt - 1) >> 1) & 1, abortp, status, 123);
            tc_fence_after_sync();
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
              uint32_t o[32];
              tmem_ld32(ocol + 32 * c, o);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_st32(ocol + 32 * c, o);
            }
            tmem_st_wait();
          }
        }
        l = fmaf(add, 0x1p-8f, l);                        // the sum is kept 2^-kSumBits times as large
        tmem_st32(scol, pk);
        tmem_st_wait();
        tc_fence_before_sync();
        mbar_arrive_warp(&sh->p_full[x][buf]);
      }
      wait_or_give_up(&sh->pv_done[x][(nk - 1) & 1], ((nk - 1) >> 1) & 1, abortp, status, 124);
      tc_fence_after_sync();
      if (!*abortp) {
        // (one factor instead of two here makes the whole loop above 10 % slower)
        const float inv = l == 0.f ? 0.f : 1.f / l, unit = 0x1p-8f / pg_top<E4M3>();
        T* dst = out + (int64_t)(e.row0 + tok) * a.nl * p.heads * p.group * D + head_row + hd * D;
        if (splits > 1 && r < valid) *reinterpret_cast<float2*>(part + (size_t)2 * PC_ROWS * D + 2 * r) = make_float2(M, l);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          tmem_ld32(ocol + 32 * c, o);
          tmem_ld_wait();
          float f[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(o[i]) * inv * unit;
          if (r < valid) {
            if (splits > 1) {
#pragma unroll
              for (int i = 0; i < 32; i += 4)
                *reinterpret_cast<float4*>(part + (size_t)r * D + 32 * c + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
            } else {
#pragma unroll
              for (int i = 0; i < 32; i += 8) store8<T>(dst + 32 * c + i, f + i);
            }
          }
        }
      }
    }
  } else if (warp < PC_SOFT_WARPS + PC_DEQ_WARPS) {
    // ---------------- codes -> operand tiles: two warps per key tile, a pair of stored tiles each ----------------
    constexpr int KP = D / 32;                            // 16-byte pieces of a lane in a stored tile
    const int dw = warp & 1, odd = (warp - PC_SOFT_WARPS) >> 1, g = lane >> 2, t = lane & 3;
    // positions of the rows of the two row tiles
    int first_pos[2], last_pos[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      first_pos[x] = base + (int)((row0 + min(x * PC_ROWS, valid - 1)) / p.group);
      last_pos[x] = base + (int)((row0 + min((x + 1) * PC_ROWS, valid) - 1) / p.group);
    }
    // lane 2 i + b knows tile b of this warp's pair in its i-th key tile of the batch, key tile batch + 2 i
    int page_l = -1, j_l = 0;
    float ak_l = 0.f, av_l = 0.f, vlast = 1.f;
    auto lookup = [&](int batch) {
      const int u = (kt0 + batch + (lane & ~1)) * PC_TILES + 2 * dw + (lane & 1);
      page_l = -1;
      j_l = 0;
      if (u < units) {
        j_l = vb.at(u) * kPageBlock;
        page_l = pg_page(p, e.seq, j_l >> p.pt_shift);
        if (page_l >= 0) {
          const float* mg = p.amax + pg_mag(p, layer, page_l, h) + (j_l & (p.pt - 1)) / kPageBlock;
          ak_l = __ldcg(mg);
          av_l = __ldcg(mg + p.pt / kPageBlock);
        }
      }
    };
    uint4 kreg[2][KP], vreg[2][KP];
    int kpage[2], kj[2];
    float kak[2], kav[2];
    // K of key tile kt on its way to registers; which piece a slot holds depends on the lane (see the stores)
    auto load = [&](int kt, bool values) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int src = (kt & 30) + b;
        const int page = __shfl_sync(0xffffffffu, page_l, src), j = __shfl_sync(0xffffffffu, j_l, src);
        const float av = __shfl_sync(0xffffffffu, av_l, src);
        if (!values) {
          kpage[b] = page;
          kj[b] = j;
          kak[b] = __shfl_sync(0xffffffffu, ak_l, src);
          kav[b] = av;
        }
        uint4(&reg)[KP] = values ? vreg[b] : kreg[b];
        // values of magnitude 0 are zeros whatever their codes are: the exponent then carries kLeastValue
        if (page >= 0 && (!values || av >= kLeastValue)) {
          const uint8_t* s = p.codes + pg_slab(p, D, layer, page, h) + (size_t)(j & (p.pt - 1)) * D + lane * 16;
          if (values) s += (size_t)p.pt * D;
#pragma unroll
          for (int i = 0; i < KP; ++i) {
            const int piece = values ? i ^ (g & 1) : (D == 128 ? i ^ (t >> 1) : i);
            reg[i] = __ldcg(reinterpret_cast<const uint4*>(s + piece * 512));
          }
          // tokens behind the end may hold any byte; a NaN code would survive its zero probability
          if (E4M3 && values && j + kPageBlock > e.len) {
            const int left = e.len - (j + 4 * t);
            const uint32_t keep = left <= 0 ? 0u : (left >= 4 ? 0xffffffffu : 0xffffffffu >> (8 * (4 - left)));
#pragma unroll
            for (int i = 0; i < KP; ++i) {
              reg[i].x &= keep;
              reg[i].y &= keep;
              reg[i].z &= keep;
              reg[i].w &= keep;
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < KP; ++i) reg[i] = make_uint4(0, 0, 0, 0);
        }
      }
    };
    lookup(odd);
    load(odd, false);
    load(odd, true);
    for (int kt = odd; kt < nk; kt += 2) {
      const int st = kt % PC_STAGES, ph = (kt / PC_STAGES) & 1;
      wait_or_give_up(&sh->k_empty[st], ph ^ 1, abortp, status, 125);
      if (__any_sync(0xffffffffu, *abortp)) break;
      unsigned char* kd = kring + st * KT;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < KP; ++i) {
          // piece j * (D / 64) + half: token 4 (g / 2) + 2 j + g % 2, dimensions t D / 4 + 16 half ..  Lanes with t >= 2
          // take the halves in the other order: then the eight lanes of a store phase hit eight different banks.
          const int j = i / (D / 64), half = D == 128 ? (i & 1) ^ (t >> 1) : 0;
          const int key = dw * 32 + (g >> 1) * 8 + b * 4 + 2 * j + (g & 1);
          const int d0 = t * (D / 4) + 16 * half;
          unsigned char* row = kd + (d0 >> 6) * (PC_KEYS * 128) + key * 128;
          const int c = (d0 & 63) >> 3;
          const uint32_t w[4] = {kreg[b][i].x, kreg[b][i].y, kreg[b][i].z, kreg[b][i].w};
          uint32_t u[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) pg_unpack4<E4M3>(w[k], u[2 * k], u[2 * k + 1]);
          *reinterpret_cast<uint4*>(row + ((c ^ (key & 7)) << 4)) = make_uint4(u[0], u[1], u[2], u[3]);
          *reinterpret_cast<uint4*>(row + (((c + 1) ^ (key & 7)) << 4)) = make_uint4(u[4], u[5], u[6], u[7]);
        }
      if (lane < 2) {
        const int b = lane, i = 2 * dw + b;
        const int page = b ? kpage[1] : kpage[0], j = b ? kj[1] : kj[0];
        const float ak = b ? kak[1] : kak[0], av = b ? kav[1] : kav[0];
        PcMeta& m = sh->meta[kt % PC_META];
        // values that are all zero may have any magnitude: the least, so that they do not set the reference of others.
        // A tile that is not there repeats the last one.
        if (page >= 0) vlast = fmaxf(av, kLeastValue);
        m.k1[i] = page >= 0 ? ak * (1.f / pg_top<E4M3>()) : 0.f;
        m.lav[i] = log2f(vlast);
        m.iav[i] = 1.f / vlast;
        m.j0[i] = page >= 0 ? j : 1 << 30;
        uint32_t part = 0;
#pragma unroll
        for (int x = 0; x < 2; ++x)
          if (page < 0 || j + kPageBlock - 1 > first_pos[x] ||
              (a.window && j <= last_pos[x] - a.window && j + kPageBlock > a.sinks))
            part |= 1u << x;
        m.part[i] = part;
      }
      fence_proxy_async_smem();
      mbar_arrive_warp(&sh->k_full[st]);
      // V of this key tile is in its registers; pages of the next batch before the next K is asked for
      if (kt + 2 < nk) {
        if (((kt + 2) & 30) == 0) lookup(kt + 2);
        load(kt + 2, false);
      }
      wait_or_give_up(&sh->v_empty[st], ph ^ 1, abortp, status, 126);
      if (__any_sync(0xffffffffu, *abortp)) break;
      unsigned char* vd = vring + st * KT;
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        // lanes with odd g take the pieces in the other order: the banks again
        const uint32_t w0[4] = {vreg[0][i].x, vreg[0][i].y, vreg[0][i].z, vreg[0][i].w};
        const uint32_t w1[4] = {vreg[1][i].x, vreg[1][i].y, vreg[1][i].z, vreg[1][i].w};
#pragma unroll
        for (int dd = 0; dd < 4; ++dd) {
          const int dim = g * (D / 8) + 4 * (i ^ (g & 1)) + dd;
          uint32_t u[4];
          pg_unpack4<E4M3>(w0[dd], u[0], u[1]);
          pg_unpack4<E4M3>(w1[dd], u[2], u[3]);
          *reinterpret_cast<uint4*>(vd + dim * 128 + (((dw * 4 + t) ^ (dim & 7)) << 4)) =
              make_uint4(u[0], u[1], u[2], u[3]);
        }
      }
      fence_proxy_async_smem();
      mbar_arrive_warp(&sh->v_full[st]);
      if (kt + 2 < nk) load(kt + 2, true);
    }
  } else if (warp == 12) {
    // ---------------- S = Q K^T ----------------
    constexpr uint32_t idesc = idesc_f16(PC_ROWS, PC_KEYS, 0, 0);
    const uint32_t on = elect_one();
    const uint64_t ad = smem_desc(smem_u32(qres), 16, 1024, kLayoutSw128);
    const uint64_t bd = smem_desc(smem_u32(kring), 16, 1024, kLayoutSw128);
    wait_or_give_up(&sh->q_full, 0, abortp, status, 127);
    float lav_most = -INFINITY;
    for (int kt = 0; kt < nk; ++kt) {
      const int st = kt % PC_STAGES;
      wait_or_give_up(&sh->k_full[st], (kt / PC_STAGES) & 1, abortp, status, 128);
      for (int x = 0; x < nx; ++x) {
        // the buffer held S and then P of key tile kt - 2
        if (kt >= 2) wait_or_give_up(&sh->pv_done[x][kt & 1], ((kt >> 1) - 1) & 1, abortp, status, 129);
        tc_fence_after_sync();
        const uint64_t a0 = desc_at(ad, x * (QT >> 4)), b0 = desc_at(bd, st * (KT >> 4));
        const uint32_t s0 = tmem + (2 * x + (kt & 1)) * PC_KEYS;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
          mma_ss_if(on, s0, desc_at(a0, (ks >> 2) * (PC_ROWS * 128 >> 4) + (ks & 3) * 2),
                    desc_at(b0, (ks >> 2) * (PC_KEYS * 128 >> 4) + (ks & 3) * 2), idesc, ks ? 1u : 0u);
        if (x == 0) {                                     // this warp meets the key tiles in order: it compares magnitudes
          const float4 lav = *reinterpret_cast<const float4*>(sh->meta[kt % PC_META].lav);
          lav_most = fmaxf(lav_most, fmaxf(fmaxf(lav.x, lav.y), fmaxf(lav.z, lav.w)));
          if (on && fminf(fminf(lav.x, lav.y), fminf(lav.z, lav.w)) < lav_most - PC_WIDE) sh->meta[kt % PC_META].part[0] = 7;
          __syncwarp();
        }
        mma_commit_if(on, &sh->s_full[x][kt & 1]);
        if (on) mbar_arrive(&sh->s_full[x][kt & 1]);      // passes on what came with k_full (the magnitudes)
        __syncwarp();
      }
      if (__any_sync(0xffffffffu, *abortp)) break;
      mma_commit_if(on, &sh->k_empty[st]);
    }
  } else {
    // ---------------- O += P V ----------------
    constexpr uint32_t idesc = idesc_f16(PC_ROWS, D, 0, 0);
    const uint32_t on = elect_one();
    const uint64_t bd = smem_desc(smem_u32(vring), 16, 1024, kLayoutSw128);
    for (int kt = 0; kt < nk; ++kt) {
      const int st = kt % PC_STAGES;
      wait_or_give_up(&sh->v_full[st], (kt / PC_STAGES) & 1, abortp, status, 130);
      for (int x = 0; x < nx; ++x) {
        wait_or_give_up(&sh->p_full[x][kt & 1], (kt >> 1) & 1, abortp, status, 131);
        tc_fence_after_sync();
        const uint64_t b0 = desc_at(bd, st * (KT >> 4));
        const uint32_t p0 = tmem + (2 * x + (kt & 1)) * PC_KEYS;
#pragma unroll
        for (int ks = 0; ks < PC_KEYS / 16; ++ks)
          mma_ts_if(on, tmem + OCOL + x * D, p0 + 8 * ks, desc_at(b0, ks * 2), idesc, (kt | ks) ? 1u : 0u);
        mma_commit_if(on, &sh->pv_done[x][kt & 1]);
      }
      if (__any_sync(0xffffffffu, *abortp)) break;
      mma_commit_if(on, &sh->v_empty[st]);
    }
  }
  drain_after_abort(abortp);
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 12) tmem_dealloc(tmem, 512);
}

// Joins the parts of split items: a warp per row of the output and head.  Part weights are l 2^(M - m), kept in fp32, the
// parts fp32 too; at most LESS_PAGES_PARTIAL_BYTES, which stay in L2.
template <typename T, int D>
__global__ void __launch_bounds__(256) pages_chunk_join_kernel(PgParams p, PaArgs a, int splits) {
  pg_wait();
  const int lane = threadIdx.x & 31, heads = a.nl * p.heads;
  const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), per_row = (int64_t)heads * p.group;
  const int row = (int)(w / per_row);
  if (row >= a.rows) return;
  const int head = (int)(w - row * per_row) / p.group, g = (int)(w - row * per_row) - head * p.group;
  int lo = 0, hi = a.n - 1;                               // the last entry that starts at or before this row
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((a.starts ? __ldg(a.starts + mid) : mid) <= row) lo = mid; else hi = mid - 1;
  }
  const PgEntry e = pg_entry(p, a.seqs, a.starts, a.rows, lo);
  if ((int64_t)e.count * p.group <= a.max_rows || row < e.row0 || row >= e.row0 + e.count) return;
  const int64_t rr = (int64_t)(row - e.row0) * p.group + g, slot = pc_slot(p, a, lo) + rr / (2 * PC_ROWS);
  const int r = (int)(rr % (2 * PC_ROWS)), c4 = (lane % (D / 4)) * 4;
  const float* part = p.partial + pc_part(slot, heads, head, splits, 0, D);
  constexpr size_t STEP = (size_t)2 * PC_ROWS * (D + 2);
  float2 ml = make_float2(-INFINITY, 0.f);
  if (lane < splits) ml = __ldcg(reinterpret_cast<const float2*>(part + lane * STEP + (size_t)2 * PC_ROWS * D + 2 * r));
  ml = pa_share(ml.x, ml.y);                              // (in the kernel before, ahead of the store, it takes 1 % of that)
  float m = ml.x;
#pragma unroll
  for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  const float weight = ml.y == 0.f ? 0.f : ml.y * pa_ex2(ml.x - m);
  float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    const float ws = __shfl_sync(0xffffffffu, weight, s);
    if (ws == 0.f) continue;                              // its values were not written
    const float4 v = __ldcg(reinterpret_cast<const float4*>(part + s * STEP + (size_t)r * D + c4));
    sum += ws;
    f.x = fmaf(ws, v.x, f.x);
    f.y = fmaf(ws, v.y, f.y);
    f.z = fmaf(ws, v.z, f.z);
    f.w = fmaf(ws, v.w, f.w);
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (lane < D / 4)
    store4(reinterpret_cast<T*>(a.out) + ((int64_t)row * per_row + (int64_t)head * p.group + g) * D + c4,
           make_float4(f.x * inv, f.y * inv, f.z * inv, f.w * inv));
}

template <typename T, int D, bool E4M3>
static int launch_chunk(const PgParams& p, const PaArgs& a, cudaStream_t s) {
  constexpr size_t smem = (size_t)(2 * PC_ROWS + 2 * PC_STAGES * PC_KEYS) * D * 2 + sizeof(PcShared);
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return fail_cuda("cudaGetDevice");
  if (dev >= 64 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
    if (cudaFuncSetAttribute(pages_chunk_kernel<T, D, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) !=
        cudaSuccess)
      return fail_cuda("shared memory opt-in of pages_chunk_kernel");
    if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  const int64_t slots = (int64_t)a.rows * p.group / (2 * PC_ROWS) + a.n, heads = (int64_t)p.heads * a.nl;
  if (slots * heads >= 0x7fffffff) return LESS_ERR_INVALID_CONFIG;
  // Items that are sure to exist; with fewer of them than multiprocessors their keys are split (measured: two sequences of
  // 30 000 tokens, eight KV heads, 48 rows each: 489 us unsplit, 82 us in nine parts)
  int64_t items = (int64_t)a.rows * p.group / (2 * PC_ROWS);
  if (items < a.n) items = a.n;
  int64_t splits = pg_sms() / (items * heads);
  const int64_t room = (int64_t)(LESS_PAGES_PARTIAL_BYTES / ((size_t)2 * PC_ROWS * (D + 2) * 4)) / (slots * heads);
  splits = splits > 32 ? 32 : splits;
  splits = splits > room ? room : splits;
  splits = splits < 1 ? 1 : splits;
  const int rc = pg_launch("pages_chunk_kernel", pages_chunk_kernel<T, D, E4M3>, dim3((unsigned)(slots * heads + 1), (unsigned)splits),
                           PC_THREADS, smem, s, p, a, (int)splits);
  if (rc != LESS_OK || splits == 1) return rc;
  const int64_t warps = (int64_t)a.rows * heads * p.group;
  return pg_launch("pages_chunk_join_kernel", pages_chunk_join_kernel<T, D>, dim3((unsigned)((warps + 7) / 8)), 256, 0, s, p, a,
                   (int)splits);
}

int launch_pages_chunk(const PgParams& p, const PaArgs& a, int dim, uint32_t flags, cudaStream_t s) {
  const bool e4m3 = flags & LESS_PAGES_E4M3;
  if (flags & LESS_PAGES_BF16) {
    if (dim == 128) return e4m3 ? launch_chunk<__nv_bfloat16, 128, true>(p, a, s) : launch_chunk<__nv_bfloat16, 128, false>(p, a, s);
    return e4m3 ? launch_chunk<__nv_bfloat16, 64, true>(p, a, s) : launch_chunk<__nv_bfloat16, 64, false>(p, a, s);
  }
  if (dim == 128) return e4m3 ? launch_chunk<__half, 128, true>(p, a, s) : launch_chunk<__half, 128, false>(p, a, s);
  return e4m3 ? launch_chunk<__half, 64, true>(p, a, s) : launch_chunk<__half, 64, false>(p, a, s);
}

}  // namespace less
