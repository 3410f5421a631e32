// The paged cache: its description on the device and what its kernels share.
#pragma once

#include "cache_index.h"
#include "common.cuh"

namespace mmshift {

// One call on a cache. Row `tok` of the call belongs to request b with
// off[b] <= tok < off[b + 1].
struct CacheJob {
  int32_t B, L, Hq, Hkv, r, d;
  int32_t bf16;                  // the call's rows are bfloat16 (else float32)
  int32_t i8;                    // the pages hold 8-bit codes with scales
  int32_t page_shift, n_pages, max_pages;
  int32_t cap;                   // positions of a sequence: max_pages << page_shift
  Divisor by_r, by_heads;        // by r and by Hkv
  int64_t stride, ls;            // elements between tokens / layers of the call's K and V, or Q
  uint8_t *kp, *vp;
  float *ks, *vs;
  const int32_t* table;
  int32_t* lens;
  int* status;
  int32_t off[MMSHIFT_MAX_BATCH + 1];
  int32_t src[MMSHIFT_MAX_BATCH + 1];   // fill: the prompts' token offsets
};

__device__ __forceinline__ int cache_request(const CacheJob& J, int tok) { return range_of(J.off, J.B, tok); }

// Rows of sequence u = (l * B + b) * Hkv + h.
__device__ __forceinline__ int cache_len(const CacheJob& J, size_t u) {
  return min(max(J.lens[u], 0), J.cap);
}

// The pool's row of position t < cap of sequence u, -1 if it has no page.
__device__ __forceinline__ int64_t cache_slot(const CacheJob& J, size_t u, int t) {
  return page_row(J.table[u * J.max_pages + (t >> J.page_shift)], J.n_pages, J.page_shift, t);
}

// Start of the cache's kernels (but the merges): everything before one in the stream is
// done, and the next one may take its place on the SMs.
__device__ __forceinline__ void cache_start() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// 16 bytes by plain loads and stores; `vec`: the address allows one access, else
// it is that of 16-bit or larger elements.
__device__ __forceinline__ uint4 load_plain16(const uint8_t* p, bool vec) {
  if (vec) return *reinterpret_cast<const uint4*>(p);
  const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
  return make_uint4(q[0] | (uint32_t)q[1] << 16, q[2] | (uint32_t)q[3] << 16,
                    q[4] | (uint32_t)q[5] << 16, q[6] | (uint32_t)q[7] << 16);
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Attention of one call: the job with Q's strides, and where results go.
struct AttendJob {
  CacheJob c;
  const uint8_t* q;
  uint8_t* out;
  float* lse;                    // or null
  int32_t causal;
  int32_t qvec, ovec;            // rows of q / out allow 16-byte accesses
  float alpha;                   // scale * log2(e)
};

size_t attend_scratch_bytes(const CacheJob& J);
cudaError_t launch_attend(const AttendJob& A, void* scratch, cudaStream_t st);

}  // namespace mmshift
