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
  const int64_t* at;             // where a sequence's entries begin in the table, or null: max_pages apart
  int32_t* lens;                 // or null: whole prompts, as many rows as the call's
  int* status;
  int32_t off[MMSHIFT_MAX_BATCH + 1];
  int32_t src[MMSHIFT_MAX_BATCH + 1];   // fill: the prompts' token offsets
};

__device__ __forceinline__ int cache_request(const CacheJob& J, int tok) { return range_of(J.off, J.B, tok); }

// Rows of sequence u = (l * B + b) * Hkv + h.
__device__ __forceinline__ int cache_len(const CacheJob& J, size_t u) {
  return min(max(J.lens[u], 0), J.cap);
}

// The page table of sequence u.
__device__ __forceinline__ const int32_t* cache_table(const CacheJob& J, size_t u) {
  return J.table + (J.at ? (size_t)J.at[u] : u * J.max_pages);
}

// The pool's row of position t < cap of sequence u, -1 if it has no page.
__device__ __forceinline__ int64_t cache_slot(const CacheJob& J, size_t u, int t) {
  return page_row(cache_table(J, u)[t >> J.page_shift], J.n_pages, J.page_shift, t);
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
  float* part;                   // or null: rows [T * Hq][d] of sums instead of out and lse, with their
  float2* part_ml;               // [T * Hq] maximum (base 2) and sum of weights, to be joined with others
  int64_t kv_stride;             // prompts: elements between two tokens' rows of K and V
  int32_t block_rows;            // prompts: rows of a block, whole tokens where a token's heads fit
  int32_t qbox;                  // prompts: Q's rows come as TMA boxes
  int32_t causal;
  int32_t qvec, ovec;            // rows of q / out allow 16-byte accesses
  float alpha;                   // scale * log2(e)
};

// Checks that the entry points share: of a call's rows, of a cache; the job of both; and of a
// workspace of a status word and `scratch` bytes more.
mmshift_status check_rows(const mmshift_shape* s);
mmshift_status check_cache(const mmshift_shape* s, const mmshift_cache* c);
mmshift_status rows_job(const mmshift_shape* s, const mmshift_cache* c, void* ws, CacheJob* J);
mmshift_status check_workspace(const void* ws, size_t bytes, size_t scratch = 0);

// What entries of attention check of their arguments, and what they make of them.
mmshift_status attend_args(const CacheJob& J, const void* Q, int64_t row_stride, int32_t causal, float softmax_scale,
                           const void* out, const float* lse);
void attend_set(AttendJob& A, const void* Q, int64_t row_stride, int32_t causal, float softmax_scale);

size_t attend_scratch_bytes(const CacheJob& J, int few = 0);
cudaError_t launch_attend(const AttendJob& A, void* scratch, cudaStream_t st);
size_t prompt_scratch_bytes(const CacheJob& J);
cudaError_t launch_prompt(AttendJob& A, void* scratch, cudaStream_t st);

}  // namespace mmshift
