// The paged cache's entry points and the kernels that write and read its rows.
//
// A row moves once: 16 bytes a lane, the lanes of a row together, K and V of a
// row by the same lanes. An 8-bit row's largest magnitude is a reduction over
// those lanes (8 to 32), so quantising costs no second pass. All three kernels
// are bound by the bytes they move, short calls by their launch.
#include <cmath>
#include <cstring>

#include "cache.cuh"

namespace mmshift {
mmshift_status noalloc_cuda_fail(cudaError_t e);
mmshift_status noalloc_prepare(const mmshift_shape* s, const mmshift_params* p, Problem* P);

namespace {

constexpr float kLeastMost = 7.703719777548943e-34f;   // 2^-110: 127 / it is finite

// The largest magnitude's bit pattern of 16 bytes of a row (8 bfloat16 or 4 float32
// values): the patterns' order is the values', and a NaN is the largest.
template <typename T>
__device__ __forceinline__ uint32_t most16(const uint4& w) {
  if constexpr (sizeof(T) == 2) {
    constexpr uint32_t k = 0x7fff7fffu;
    const uint32_t m = __vmaxu2(__vmaxu2(w.x & k, w.y & k), __vmaxu2(w.z & k, w.w & k));
    return max(m & 0xffffu, m >> 16);
  } else {
    constexpr uint32_t k = 0x7fffffffu;
    return max(max(w.x & k, w.y & k), max(w.z & k, w.w & k));
  }
}

// rint(x * inv), at most 127 (1 + 2^-23) before it is rounded: 1.5 * 2^23 added, the sum's
// last byte is the code (no conversion: those go at a quarter of the rate).
template <typename T>
__device__ __forceinline__ void codes16(const uint4& w, float inv, uint32_t (&code)[2]) {
  constexpr int N = 16 / (int)sizeof(T);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  uint32_t c[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float x;
    if constexpr (sizeof(T) == 2) x = (i & 1) ? bf16_hi(u[i / 2]) : bf16_lo(u[i / 2]);
    else x = __uint_as_float(u[i]);
    c[i] = __float_as_uint(__fadd_rn(__fmul_rn(x, inv), 12582912.f));
  }
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const uint32_t lo = __byte_perm(c[i], c[i + 1], 0x0040), hi = __byte_perm(c[i + 2], c[i + 3], 0x0040);
    code[i / 4] = inv != 0.f ? __byte_perm(lo, hi, 0x5410) : 0;   // x may be no number
  }
}

// The codes of 16 bytes of a K and of a V row, by the LPR lanes that hold them, and
// their scale: K's in lanes 2, 6, ..., V's in lanes 3, 7, ... Of a row pair's four quotients
// every lane works out one: with all four, a reduction for each row and conversions,
// filling 229,000 bfloat16 rows and reading them back took 73.5 us instead of 69.
template <typename T, int LPR>
__device__ __forceinline__ float quantise16(const uint4& k, const uint4& v, int part, uint32_t (&ck)[2],
                                            uint32_t (&cv)[2]) {
  uint32_t mk = most16<T>(k), mv = most16<T>(v);
  if constexpr (sizeof(T) == 2) {
    uint32_t m = mk | mv << 16;
#pragma unroll
    for (int s = LPR / 2; s; s >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, s));
    mk = m << 16;
    mv = m & 0xffff0000u;
  } else {
#pragma unroll
    for (int s = LPR / 2; s; s >>= 1) {
      mk = max(mk, __shfl_xor_sync(0xffffffffu, mk, s));
      mv = max(mv, __shfl_xor_sync(0xffffffffu, mv, s));
    }
  }
  const uint32_t m = part & 1 ? mv : mk;
  const float most = __uint_as_float(m), q = __fdiv_rn(part & 2 ? most : 127.f, part & 2 ? 127.f : most);
  auto usable = [](uint32_t x) { return x < 0x7f800000u && __uint_as_float(x) >= kLeastMost; };
  const float ik = __shfl_sync(0xffffffffu, q, 0, LPR), iv = __shfl_sync(0xffffffffu, q, 1, LPR);
  codes16<T>(k, usable(mk) ? ik : 0.f, ck);
  codes16<T>(v, usable(mv) ? iv : 0.f, cv);
  return m < 0x7f800000u ? q : __uint_as_float(0x7fffffffu);
}

// Rows into pages. FILL: the rows idx keeps of a prompt, to positions 0, 1, ...;
// else a call's own rows, to the last positions of their sequences. A group of lanes
// takes N rows, whose table entries, then whose data are all asked for before any is
// used: a row's chain of loads (length or index, table, data) is as long as its
// store's, and with one row a group the memory waits (see kMany).
template <typename T, int D, bool I8, bool FILL, int N>
__global__ void __launch_bounds__(256) cache_write_kernel(const __grid_constant__ CacheJob J,
                                                          const uint8_t* K, const uint8_t* V,
                                                          const int32_t* idx, const int32_t* count,
                                                          bool vec) {
  cache_start();
  constexpr int ROWB = D * (int)sizeof(T), LPR = ROWB / 16, G = 256 / LPR;
  const int l = blockIdx.y, part = threadIdx.x % LPR;
  const int rows = J.off[J.B] * J.Hkv;                    // at most 2^30
  const int64_t q0 = (int64_t)blockIdx.x * (G * N) + threadIdx.x / LPR;
  int pos[N], entry[N];
  bool there[N], bad[N];
  size_t src[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const bool live = q0 + k * G < rows;                  // all lanes stay for the reduction
    const int q = live ? (int)(q0 + k * G) : 0, c = J.by_heads(q), h = q - c * J.Hkv;
    const int b = cache_request(J, c), i = c - J.off[b], n = J.off[b + 1] - J.off[b];
    const size_t u = ((size_t)l * J.B + b) * J.Hkv + h;
    bad[k] = false;
    if constexpr (FILL) {
      const int m = live && count ? min(max(count[u], 0), n) : n;
      if (live && part == 0 && i == 0) J.lens[u] = min(m, J.cap);
      pos[k] = i;
      there[k] = live && i < m;
      const int t = there[k] ? idx[(size_t)l * rows + q] : 0;
      bad[k] = there[k] && (t < 0 || t >= J.src[b + 1] - J.src[b]);
      src[k] = ((size_t)l * J.ls + (((size_t)J.src[b] + (bad[k] ? 0 : t)) * J.Hkv + h) * D) * sizeof(T);
    } else {
      pos[k] = live ? append_end(J.lens[u], J.cap) - n + i : 0;
      there[k] = live && pos[k] >= 0;
      src[k] = ((size_t)l * J.ls + (size_t)c * J.stride + (size_t)h * D) * sizeof(T);
    }
    entry[k] = there[k] && pos[k] < J.cap ? J.table[u * J.max_pages + (pos[k] >> J.page_shift)] : -1;
  }
  uint4 kk[N], vv[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    kk[k] = vv[k] = make_uint4(0, 0, 0, 0);
    if (there[k] && !bad[k]) {                            // an input row, whether its page is there or not
      kk[k] = load_plain16(K + src[k] + part * 16, vec);
      vv[k] = load_plain16(V + src[k] + part * 16, vec);
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int64_t slot = page_row(entry[k], J.n_pages, J.page_shift, pos[k]);
    if (there[k] && part == 0) {
      if (bad[k]) set_status(J.status, kStatusBadIndex);
      if (slot < 0) set_status(J.status, kStatusBadPage);
    }
    if constexpr (I8) {
      uint32_t ck[2], cv[2];
      const float scale = quantise16<T, LPR>(kk[k], vv[k], part, ck, cv);
      if (slot < 0) continue;
      constexpr int CB = 16 / (int)sizeof(T);             // code bytes of a lane
      const size_t dst = (size_t)slot * D + part * CB;
      if constexpr (CB == 8) {
        *reinterpret_cast<uint2*>(J.kp + dst) = make_uint2(ck[0], ck[1]);
        *reinterpret_cast<uint2*>(J.vp + dst) = make_uint2(cv[0], cv[1]);
      } else {
        *reinterpret_cast<uint32_t*>(J.kp + dst) = ck[0];
        *reinterpret_cast<uint32_t*>(J.vp + dst) = cv[0];
      }
      if (part == 2) J.ks[slot] = scale;
      if (part == 3) J.vs[slot] = scale;
    } else {
      if (slot < 0) continue;
      const size_t dst = (size_t)slot * ROWB + part * 16;
      *reinterpret_cast<uint4*>(J.kp + dst) = kk[k];
      *reinterpret_cast<uint4*>(J.vp + dst) = vv[k];
    }
  }
}

// What lies in a page of the 16 bytes of an output row at `part`, and those bytes.
template <typename T, int D, bool I8>
struct PageRow {
  static constexpr int N = 16 / (int)sizeof(T);
  uint32_t w[I8 ? N / 4 : 4];
  float s;
  __device__ __forceinline__ void load(const uint8_t* pages, const float* scales, int64_t slot, int part) {
    if constexpr (!I8) {
      const uint4 v = *reinterpret_cast<const uint4*>(pages + (size_t)slot * D * sizeof(T) + part * 16);
      w[0] = v.x;
      w[1] = v.y;
      w[2] = v.z;
      w[3] = v.w;
    } else {
      const uint8_t* p = pages + (size_t)slot * D + part * N;
      if constexpr (N == 8) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[0] = v.x;
        w[1] = v.y;
      } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
      }
      s = scales[slot];
    }
  }
  __device__ __forceinline__ uint4 value() const {
    if constexpr (!I8) {
      return make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      float x[N];
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = (float)(int8_t)(w[i / 4] >> (8 * (i & 3))) * s;
      if constexpr (N == 8)
        return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                          pack_bf16(x[6], x[7]));
      else
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                          __float_as_uint(x[3]));
    }
  }
};

// Rows of pages back out, N of them a group of lanes as in cache_write_kernel.
template <typename T, int D, bool I8, int N>
__global__ void __launch_bounds__(256) cache_read_kernel(const __grid_constant__ CacheJob J,
                                                         const int32_t* first, uint8_t* oK,
                                                         uint8_t* oV, bool vec) {
  cache_start();
  constexpr int ROWB = D * (int)sizeof(T), LPR = ROWB / 16, G = 256 / LPR;
  const int l = blockIdx.y, part = threadIdx.x % LPR;
  const int rows = J.off[J.B] * J.Hkv;
  const int64_t q0 = (int64_t)blockIdx.x * (G * N) + threadIdx.x / LPR;
  int pos[N], entry[N];
  bool in[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const bool live = q0 + k * G < rows;
    const int q = live ? (int)(q0 + k * G) : 0, c = J.by_heads(q), h = q - c * J.Hkv;
    const int b = cache_request(J, c);
    const size_t u = ((size_t)l * J.B + b) * J.Hkv + h;
    const int64_t t = (int64_t)(c - J.off[b]) + (first ? first[u] : 0);
    in[k] = live && t >= 0 && t < cache_len(J, u);
    pos[k] = in[k] ? (int)t : 0;
    entry[k] = in[k] ? J.table[u * J.max_pages + (pos[k] >> J.page_shift)] : -1;
  }
  PageRow<T, D, I8> kr[N], vr[N];
  bool there[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int64_t slot = page_row(entry[k], J.n_pages, J.page_shift, pos[k]);
    there[k] = slot >= 0;
    if (there[k]) {
      kr[k].load(J.kp, J.ks, slot, part);
      vr[k].load(J.vp, J.vs, slot, part);
    } else if (in[k] && part == 0) {
      set_status(J.status, kStatusBadPage);
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int64_t q = q0 + k * G;
    if (q >= rows) continue;
    const size_t dst = ((size_t)l * rows + q) * ROWB + part * 16;
    const uint4 none = make_uint4(0, 0, 0, 0);
    store_row16(oK + dst, there[k] ? kr[k].value() : none, vec);
    store_row16(oV + dst, there[k] ? vr[k].value() : none, vec);
  }
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace

mmshift_status check_cache(const mmshift_shape* s, const mmshift_cache* c) {
  if (!c) return MMSHIFT_ERR_INVALID_ARG;
  if (c->dtype != s->dtype && c->dtype != MMSHIFT_I8) return MMSHIFT_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
    return MMSHIFT_ERR_UNSUPPORTED;
  if (c->n_pages < 1 || c->max_pages < 1) return MMSHIFT_ERR_INVALID_ARG;
  if ((int64_t)c->n_pages * c->page_size >= (int64_t)INT32_MAX - 256 ||
      (int64_t)c->max_pages * c->page_size > (int64_t)1 << 30)
    return MMSHIFT_ERR_UNSUPPORTED;
  if (!c->k_pages || !c->v_pages || !c->page_table || !c->lens) return MMSHIFT_ERR_INVALID_ARG;
  if (!aligned(c->k_pages, 16) || !aligned(c->v_pages, 16) || !aligned(c->page_table, 4) || !aligned(c->lens, 4))
    return MMSHIFT_ERR_INVALID_ARG;
  if (c->dtype == MMSHIFT_I8 &&
      (!c->k_scales || !c->v_scales || !aligned(c->k_scales, 4) || !aligned(c->v_scales, 4)))
    return MMSHIFT_ERR_INVALID_ARG;
  return MMSHIFT_OK;
}

// The shape of a call on a cache: its rows, some requests without any.
mmshift_status check_rows(const mmshift_shape* s) {
  if (!s || !s->cu_seqlens) return MMSHIFT_ERR_INVALID_ARG;
  if (s->batch < 1 || s->batch > MMSHIFT_MAX_BATCH) return MMSHIFT_ERR_INVALID_ARG;
  if (s->n_layers < 1 || s->n_layers > MMSHIFT_MAX_LAYERS) return MMSHIFT_ERR_INVALID_ARG;
  if (s->n_kv_heads < 1 || s->n_q_heads < s->n_kv_heads || s->n_q_heads % s->n_kv_heads)
    return MMSHIFT_ERR_INVALID_ARG;
  if (s->dtype != MMSHIFT_BF16 && s->dtype != MMSHIFT_F32) return MMSHIFT_ERR_UNSUPPORTED;
  if (s->head_dim != 64 && s->head_dim != 128) return MMSHIFT_ERR_UNSUPPORTED;
  if (s->cu_seqlens[0] != 0) return MMSHIFT_ERR_INVALID_ARG;
  for (int b = 0; b < s->batch; ++b)
    if (s->cu_seqlens[b + 1] < s->cu_seqlens[b]) return MMSHIFT_ERR_INVALID_ARG;
  // a layer's sequences, and rows of all heads, are counted in 31 bits of blocks and of indices
  if ((int64_t)s->batch * s->n_kv_heads > (int64_t)1 << 30) return MMSHIFT_ERR_UNSUPPORTED;
  if ((int64_t)s->cu_seqlens[s->batch] * s->n_q_heads > (int64_t)1 << 30) return MMSHIFT_ERR_UNSUPPORTED;
  return MMSHIFT_OK;
}

static void fill_job(const mmshift_shape* s, const mmshift_cache* c, void* ws, CacheJob* J) {
  std::memset(J, 0, sizeof(*J));
  J->B = s->batch;
  J->L = s->n_layers;
  J->Hq = s->n_q_heads;
  J->Hkv = s->n_kv_heads;
  J->r = s->n_q_heads / s->n_kv_heads;
  J->by_r = divisor_of(J->r);
  J->by_heads = divisor_of(J->Hkv);
  J->d = s->head_dim;
  J->bf16 = s->dtype == MMSHIFT_BF16;
  J->i8 = c->dtype == MMSHIFT_I8;
  while ((1 << J->page_shift) < c->page_size) ++J->page_shift;
  J->n_pages = c->n_pages;
  J->max_pages = c->max_pages;
  J->cap = c->max_pages << J->page_shift;
  J->kp = static_cast<uint8_t*>(c->k_pages);
  J->vp = static_cast<uint8_t*>(c->v_pages);
  J->ks = c->k_scales;
  J->vs = c->v_scales;
  J->table = c->page_table;
  J->lens = c->lens;
  J->status = static_cast<int*>(ws);
}

mmshift_status rows_job(const mmshift_shape* s, const mmshift_cache* c, void* ws, CacheJob* J) {
  mmshift_status st = check_rows(s);
  if (st == MMSHIFT_OK) st = check_cache(s, c);
  if (st != MMSHIFT_OK) return st;
  fill_job(s, c, ws, J);
  for (int b = 0; b <= s->batch; ++b) J->off[b] = s->cu_seqlens[b];
  return MMSHIFT_OK;
}

mmshift_status attend_args(const CacheJob& J, const void* Q, int64_t row_stride, int32_t causal, float softmax_scale,
                           const void* out, const float* lse) {
  const size_t esz = J.bf16 ? 2 : 4;
  if (row_stride && row_stride < (int64_t)J.Hq * J.d) return MMSHIFT_ERR_INVALID_ARG;
  if (causal != 0 && causal != 1) return MMSHIFT_ERR_INVALID_ARG;
  if (!(softmax_scale >= 0.f) || !std::isfinite(softmax_scale * kLog2e)) return MMSHIFT_ERR_INVALID_ARG;
  if (J.off[J.B] && (!Q || !out)) return MMSHIFT_ERR_INVALID_ARG;
  if (!aligned(Q, esz) || !aligned(out, esz) || !aligned(lse, 4)) return MMSHIFT_ERR_INVALID_ARG;
  return MMSHIFT_OK;
}

void attend_set(AttendJob& A, const void* Q, int64_t row_stride, int32_t causal, float softmax_scale) {
  CacheJob& J = A.c;
  J.stride = row_stride ? row_stride : (int64_t)J.Hq * J.d;
  A.q = static_cast<const uint8_t*>(Q);
  A.causal = causal;
  A.qvec = aligned(Q, 16) && J.stride * (J.bf16 ? 2 : 4) % 16 == 0;
  A.alpha = (softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)J.d)) * kLog2e;
}

// Rows are moved with the status word alone, attention takes `scratch` bytes more.
mmshift_status check_workspace(const void* ws, size_t bytes, size_t scratch) {
  return ws && aligned(ws, 256) && bytes >= 256 + scratch ? MMSHIFT_OK : MMSHIFT_ERR_WORKSPACE;
}

namespace {

// Calls of more rows (of all heads and layers) than this give each group of lanes four to
// read, or two to write: 609,000 8-bit rows are read in 74.2 us instead of 87.3 (6.4 TB/s);
// 229,000 written, 8-bit from bfloat16, and read back in 65 (68 with one row written, 69
// with four, 88 with eight), unquantised float32 in 72 (76, 73). 17,800 rows take 15.9
// instead of 9.7 us with four, 3,076 float32 rows 3.7 instead of 2.7.
constexpr int64_t kMany = 40000;

template <bool FILL, int N>
cudaError_t launch_write_n(const CacheJob& J, const void* K, const void* V, const int32_t* idx,
                           const int32_t* count, cudaStream_t st) {
  const int esz = J.bf16 ? 2 : 4, per = N * 256 / (J.d * esz / 16);
  const bool vec = aligned(K, 16) && aligned(V, 16) && J.stride * esz % 16 == 0 && J.ls * esz % 16 == 0;
  const dim3 grid((unsigned)(((int64_t)J.off[J.B] * J.Hkv + per - 1) / per), J.L);
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, grid, 256, 0, st, true, 0, J, (const uint8_t*)K, (const uint8_t*)V, idx,
                         count, vec);
  };
  if (J.bf16) {
    if (J.d == 128)
      return J.i8 ? go(cache_write_kernel<__nv_bfloat16, 128, true, FILL, N>)
                  : go(cache_write_kernel<__nv_bfloat16, 128, false, FILL, N>);
    return J.i8 ? go(cache_write_kernel<__nv_bfloat16, 64, true, FILL, N>)
                : go(cache_write_kernel<__nv_bfloat16, 64, false, FILL, N>);
  }
  if (J.d == 128)
    return J.i8 ? go(cache_write_kernel<float, 128, true, FILL, N>) : go(cache_write_kernel<float, 128, false, FILL, N>);
  return J.i8 ? go(cache_write_kernel<float, 64, true, FILL, N>) : go(cache_write_kernel<float, 64, false, FILL, N>);
}

template <bool FILL>
cudaError_t launch_write(const CacheJob& J, const void* K, const void* V, const int32_t* idx,
                         const int32_t* count, cudaStream_t st) {
  const int64_t rows = (int64_t)J.off[J.B] * J.Hkv * J.L;
  if (!rows) return cudaSuccess;
  return rows > kMany ? launch_write_n<FILL, 2>(J, K, V, idx, count, st)
                      : launch_write_n<FILL, 1>(J, K, V, idx, count, st);
}

template <int N>
cudaError_t launch_read_n(const CacheJob& J, const int32_t* first, void* oK, void* oV, cudaStream_t st) {
  const int esz = J.bf16 ? 2 : 4, per = N * 256 / (J.d * esz / 16);
  const bool vec = aligned(oK, 16) && aligned(oV, 16);
  const dim3 grid((unsigned)(((int64_t)J.off[J.B] * J.Hkv + per - 1) / per), J.L);
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, grid, 256, 0, st, true, 0, J, first, (uint8_t*)oK, (uint8_t*)oV, vec);
  };
  if (J.bf16) {
    if (J.d == 128)
      return J.i8 ? go(cache_read_kernel<__nv_bfloat16, 128, true, N>) : go(cache_read_kernel<__nv_bfloat16, 128, false, N>);
    return J.i8 ? go(cache_read_kernel<__nv_bfloat16, 64, true, N>) : go(cache_read_kernel<__nv_bfloat16, 64, false, N>);
  }
  if (J.d == 128)
    return J.i8 ? go(cache_read_kernel<float, 128, true, N>) : go(cache_read_kernel<float, 128, false, N>);
  return J.i8 ? go(cache_read_kernel<float, 64, true, N>) : go(cache_read_kernel<float, 64, false, N>);
}

cudaError_t launch_read(const CacheJob& J, const int32_t* first, void* oK, void* oV, cudaStream_t st) {
  const int64_t rows = (int64_t)J.off[J.B] * J.Hkv * J.L;
  if (!rows) return cudaSuccess;
  return rows > kMany ? launch_read_n<4>(J, first, oK, oV, st) : launch_read_n<1>(J, first, oK, oV, st);
}

mmshift_status done(cudaError_t e) { return e == cudaSuccess ? MMSHIFT_OK : noalloc_cuda_fail(e); }

}  // namespace
}  // namespace mmshift

using namespace mmshift;

extern "C" {

mmshift_status mmshift_cache_workspace_size(const mmshift_shape* s, const mmshift_cache* c,
                                            size_t* bytes) {
  CacheJob J;
  const mmshift_status st = rows_job(s, c, nullptr, &J);
  if (st != MMSHIFT_OK) return st;
  if (!bytes) return MMSHIFT_ERR_INVALID_ARG;
  *bytes = 256 + attend_scratch_bytes(J);
  return MMSHIFT_OK;
}

mmshift_status mmshift_cache_fill(const mmshift_shape* s, const mmshift_cache* c, const void* K,
                                  const void* V, const int32_t* idx, const int32_t* count,
                                  void* workspace, size_t workspace_bytes,
                                  mmshift_stream_t stream) {
  Problem P;
  mmshift_status st = noalloc_prepare(s, nullptr, &P);
  if (st == MMSHIFT_OK) st = check_cache(s, c);
  if (st != MMSHIFT_OK) return st;
  const size_t esz = s->dtype == MMSHIFT_BF16 ? 2 : 4;
  if (!K || !V || !idx || !aligned(K, esz) || !aligned(V, esz) || !aligned(idx, 4) || !aligned(count, 4))
    return MMSHIFT_ERR_INVALID_ARG;
  if ((int64_t)P.R * P.Hkv > (int64_t)1 << 30) return MMSHIFT_ERR_UNSUPPORTED;
  CacheJob J;
  fill_job(s, c, workspace, &J);
  for (int b = 0; b < P.B; ++b) {
    J.off[b] = P.req[b].out_off;
    J.src[b + 1] = P.req[b].tok_off + P.req[b].t_len;
  }
  J.off[P.B] = P.R;
  J.ls = P.ls_kv;
  if ((st = check_workspace(workspace, workspace_bytes)) != MMSHIFT_OK) return st;
  if (!device_readable(K) || !device_readable(V)) return MMSHIFT_ERR_INVALID_ARG;
  return done(launch_write<true>(J, K, V, idx, count, (cudaStream_t)stream));
}

mmshift_status mmshift_cache_append(const mmshift_shape* s, const mmshift_cache* c, const void* K,
                                    const void* V, int64_t row_stride, void* workspace,
                                    size_t workspace_bytes, mmshift_stream_t stream) {
  CacheJob J;
  mmshift_status st = rows_job(s, c, workspace, &J);
  if (st != MMSHIFT_OK) return st;
  const size_t esz = J.bf16 ? 2 : 4;
  const int64_t dense = (int64_t)J.Hkv * J.d, total = J.off[J.B];
  if (row_stride && row_stride < dense) return MMSHIFT_ERR_INVALID_ARG;
  J.stride = row_stride ? row_stride : dense;
  J.ls = J.L > 1 ? s->layer_stride_kv : 0;
  if (J.L > 1 && total && J.ls < (total - 1) * J.stride + dense) return MMSHIFT_ERR_INVALID_ARG;
  if (total && (!K || !V)) return MMSHIFT_ERR_INVALID_ARG;
  if (!aligned(K, esz) || !aligned(V, esz)) return MMSHIFT_ERR_INVALID_ARG;
  if ((st = check_workspace(workspace, workspace_bytes)) != MMSHIFT_OK) return st;
  return done(launch_write<false>(J, K, V, nullptr, nullptr, (cudaStream_t)stream));
}

mmshift_status mmshift_cache_read(const mmshift_shape* s, const mmshift_cache* c,
                                  const int32_t* first, void* out_K, void* out_V, void* workspace,
                                  size_t workspace_bytes, mmshift_stream_t stream) {
  CacheJob J;
  mmshift_status st = rows_job(s, c, workspace, &J);
  if (st != MMSHIFT_OK) return st;
  const size_t esz = J.bf16 ? 2 : 4;
  if (J.off[J.B] && (!out_K || !out_V)) return MMSHIFT_ERR_INVALID_ARG;
  if (!aligned(out_K, esz) || !aligned(out_V, esz) || !aligned(first, 4)) return MMSHIFT_ERR_INVALID_ARG;
  if ((st = check_workspace(workspace, workspace_bytes)) != MMSHIFT_OK) return st;
  return done(launch_read(J, first, out_K, out_V, (cudaStream_t)stream));
}

mmshift_status mmshift_cache_attention(const mmshift_shape* s, const mmshift_cache* c,
                                       const void* Q, int64_t row_stride, int32_t causal,
                                       float softmax_scale, void* out, float* lse,
                                       void* workspace, size_t workspace_bytes,
                                       mmshift_stream_t stream) {
  AttendJob A;
  std::memset(&A, 0, sizeof(A));
  CacheJob& J = A.c;
  mmshift_status st = rows_job(s, c, workspace, &J);
  if (st != MMSHIFT_OK) return st;
  if (J.L != 1) return MMSHIFT_ERR_UNSUPPORTED;
  if ((st = attend_args(J, Q, row_stride, causal, softmax_scale, out, lse)) != MMSHIFT_OK) return st;
  if ((st = check_workspace(workspace, workspace_bytes, attend_scratch_bytes(J))) != MMSHIFT_OK) return st;
  attend_set(A, Q, row_stride, causal, softmax_scale);
  A.out = static_cast<uint8_t*>(out);
  A.ovec = aligned(out, 16);
  A.lse = lse;
  if (!J.off[J.B]) return MMSHIFT_OK;
  return done(launch_attend(A, static_cast<char*>(workspace) + 256, (cudaStream_t)stream));
}

}  // extern "C"
