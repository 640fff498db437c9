// The paged 8-bit cache: parameters, index arithmetic, the stored tile order and the code formats, shared by
// pages_ops.cu (maps and page moves), pages_write.cu and pages_attn.cu.
//
// Order of a tile (16 tokens x D dimensions of one head, 16 * D bytes).  A tile lies in memory as a warp consumes
// it: 16-byte pieces, piece = 32 * c + 4 * g + t of lane (g = lane / 4, t = lane % 4), so that a warp-wide 16-byte
// load is 512 contiguous bytes and what a lane loads is what its m16n8k16 operand fragments hold:
//   keys    c = j * (D / 64) + half:  token 4 (g / 2) + 2 j + g % 2, dimensions t * D / 4 + 16 half .. + 15
//   values  c = i:                    dimensions g * D / 8 + 4 i .. + 3, each the tokens 4 t .. 4 t + 3
// (the scores' accumulators come out as tokens x rows; the permuted token order above makes a value word's four
// tokens the four reduction indices 2t, 2t + 1, 2t + 8, 2t + 9 that the lane supplies to the second product).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "less_internal.cuh"

namespace less {

constexpr int kPageBlock = LESS_PAGE_BLOCK;      // tokens that share a magnitude

// status word values of the cache (first writer wins; see less_pages_poll_status)
constexpr int kPagesBounds = 2, kPagesExhausted = 3, kPagesState = 4;

struct PgParams {
  int layers, heads, group, pt, pt_shift, pages, seqs, seq_pages;
  uint8_t* codes;
  float* amax;
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  int32_t* status;         // [4] first words of the workspace: code and place of an error; of an error of write or trim
  int32_t* moves;          // [0] number of page moves of the call under way, then (source, destination) of each
  int32_t* mark;           // [seqs]
  int32_t* off;            // [seqs]
  int32_t* fresh;          // [max(seqs, pages)]
  int32_t* counters;       // [kPgCounters] zero between calls
  float* partial;          // partial results of the step kernel
};

constexpr int kPgCounters = 1024;

__device__ __forceinline__ void pg_status(int32_t* status, int code, int where) {
  if (atomicCAS(status, 0, code) == 0) status[1] = where;
}

// Write and trim run on many CTAs, some of which find errors while others have not begun.  So that what they do does not
// depend on which is first, they look at the first word and report to the second: an entry that is refused stops no other
// one.  A call that is planned by one CTA sees both, and moves the second to the first.
constexpr int kLateStatus = 2;
__device__ __forceinline__ bool pg_stopped(const PgParams& p) {
  const int4 s = __ldcg(reinterpret_cast<const int4*>(p.status));
  if (s.z && threadIdx.x == 0) pg_status(p.status, s.z, s.w);
  return (s.x | s.z) != 0;
}

__host__ __device__ __forceinline__ int pg_ceil(int a, int b) { return (a + b - 1) / b; }

// first code byte of (layer, page, head); the keys' tiles, then the values'
__device__ __forceinline__ size_t pg_slab(const PgParams& p, int D, int layer, int page, int head) {
  return (((size_t)layer * p.pages + page) * p.heads + head) * ((size_t)2 * p.pt * D);
}
// first magnitude of (layer, page, head): pt / 16 of the keys, then of the values
__device__ __forceinline__ size_t pg_mag(const PgParams& p, int layer, int page, int head) {
  return (((size_t)layer * p.pages + page) * p.heads + head) * ((size_t)2 * (p.pt / kPageBlock));
}

template <bool E4M3>
__host__ __device__ constexpr float pg_top() { return E4M3 ? 448.f : 127.f; }

// four codes -> two packed pairs of fp16, exactly.  int8: the code with its sign bit flipped is the low byte of the
// fp16 number 1024 + (code + 128); subtracting 1152 leaves the code.  e4m3: the hardware conversion.
template <bool E4M3>
__device__ __forceinline__ void pg_unpack4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (E4M3) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
  } else {
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const uint32_t bias = 0x64806480u;
    const __half2 ra = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&bias));
    const __half2 rb = __hsub2(*reinterpret_cast<const __half2*>(&b), *reinterpret_cast<const __half2*>(&bias));
    lo = *reinterpret_cast<const uint32_t*>(&ra);
    hi = *reinterpret_cast<const uint32_t*>(&rb);
  }
}

// a length that the caller has overwritten with something else must not become an address
__device__ __forceinline__ bool pg_len_ok(const PgParams& p, int len) { return len >= 0 && len <= p.seq_pages * p.pt; }

// The entries of a call: entry i is the sequence seqs[i] with `count` new tokens, rows [row0, row0 + count) of the
// call's inputs, at positions [len - count, len).  An index out of range counts as an entry without tokens.
struct PgEntry {
  int seq, row0, count, len;
};
__device__ __forceinline__ PgEntry pg_entry(const PgParams& p, const int32_t* seqs, const int32_t* starts, int rows,
                                            int i) {
  PgEntry e;
  e.seq = __ldg(seqs + i);
  e.row0 = starts ? __ldg(starts + i) : i;
  const int end = starts ? __ldg(starts + i + 1) : i + 1;
  e.len = 0;
  e.count = 0;
  if (e.seq < 0 || e.seq >= p.seqs || e.row0 < 0 || end < e.row0 || end > rows) {
    pg_status(p.status, kPagesBounds, 1);
    e.seq = 0;
    e.row0 = 0;
  } else {
    e.count = end - e.row0;
    e.len = __ldcg(p.lens + e.seq);
    if (!pg_len_ok(p, e.len)) {
      pg_status(p.status, kPagesBounds, 2);
      e.len = 0;
      e.count = 0;
    }
  }
  return e;
}

// Whether entry i starts behind its end.  Kernels that look entries up by their rows miss some then, so one CTA of them
// looks at all.
__device__ __forceinline__ bool pg_descends(const int32_t* starts, int i) { return starts && __ldg(starts + i + 1) < __ldg(starts + i); }
__device__ __forceinline__ void pg_check_starts(const PgParams& p, const int32_t* starts, int n) {
  for (int i = threadIdx.x; i < n; i += blockDim.x)
    if (pg_descends(starts, i)) pg_status(p.status, kPagesBounds, 4);
}

// page of the tokens [ordinal * pt, + pt) of a sequence, -1 = none
__device__ __forceinline__ int pg_page(const PgParams& p, int seq, int ordinal) {
  const int page = __ldcg(p.table + (size_t)seq * p.seq_pages + ordinal);
  if (page >= p.pages) {
    pg_status(p.status, kPagesBounds, 3);
    return -1;
  }
  return page;
}

// Every kernel of the cache is launched as a programmatic dependent of the kernel before it in the stream: its CTAs come
// up while that one drains and wait, before they read anything, until it is complete (pg_wait).  Each lets its own
// dependents come up once all its CTAs run.  So a kernel may be on an SM whose L1 still takes lines for the one before:
// whatever a kernel of the cache writes (maps, codes, magnitudes, partial results) is read past L1, with __ldcg.
__device__ __forceinline__ void pg_wait() {
  pdl_wait_primary();
  pdl_launch_dependents();
}

template <typename... P, typename... A>
inline int pg_launch(const char* name, void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
  return e == cudaSuccess ? check_launch(name) : fail_cuda(name, e);
}

// host: checks a description; on success fills the device view
int pg_view(const less_pages* d, PgParams* p);
int pg_sms();

}  // namespace less
