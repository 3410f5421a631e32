// Attention of float32 rows, over float32 or 8-bit pages: CUDA cores, fp32 FMAs.
//
// Tiles of NT / 16 * TR query rows over tiles of BK keys: thread (ty, tx) has the TR rows of
// group ty; in S the keys tx, tx + 16, ..., in O the dimensions 4 tx .. of each 64. A row's
// threads are 16 lanes of one warp, so its weights change hands through shared memory
// without a barrier of the CTA. K of the next tile arrives (asynchronous copies; 8-bit
// codes through registers, to be converted) while this one's values are added up, V while
// its logits are. The shape follows from what shared memory feeds the FMAs, 128 bytes
// a clock and SM. Chunks (NT = 256, TR = 8: 128 rows by 64 keys): 8 x 4 sums take 1.5 bytes
// an FMA, the 8 x 8 (or 8 x 4, d = 64) of the second product 1 (1.5): 512 tokens of 28
// heads over 4096 rows, d = 128, 607 us (46 TFLOP/s of 80). Counters there: FMA pipe 65 % of
// cycles, shared memory 53 %, issue slots 45 % (d = 64, 257 tokens: 52, 40, 41 %): 250 registers
// leave two warps a scheduler, which mostly wait out an instruction's latency. Few rows (TR = 2, two or four
// warps, five or four CTAs an SM): 64 requests of one token, 64 heads, 500 to 6000 rows
// 312 us (4.9 TB/s) over float32 pages, 350 over 8-bit ones; 445 and 451 with four warps
// and TR = 1, which read a key four times, not twice; 334 and 452 with one warp and TR = 4, too
// few to hide the loads.
#include <type_traits>

#include "attend.cuh"
#include "umma.cuh"

namespace mmshift {
namespace {

using umma::ffma2;
using umma::lds_2x64;
using umma::pk2;
using umma::smem_u32;
using umma::upk2;

constexpr float kRaise = 8.f;

template <int D, int NT, int TR>
struct Simt {
  static constexpr int BK = NT == 256 ? 64 : 32, NK = BK / 16;
  static constexpr int RT = NT / 16 * TR;
  static constexpr int QS = D + 4, PS = RT + 4;        // floats between rows: no bank conflicts
  struct Smem {
    alignas(16) float q[RT][QS];
    alignas(16) float k[BK][QS];
    alignas(16) float v[BK][D];
    alignas(16) float p[BK][PS];
    float ks[BK], vs[BK];
    AttendScan<NT, 512> scan;
  };
};

__device__ __forceinline__ void copy16(void* dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(in ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

// Four codes as floats: 2^23 + 128 + code has the code's bits, the sign's turned over, at its
// end, so that no conversion is needed.
__device__ __forceinline__ float4 codes4(uint32_t x) {
  x ^= 0x80808080u;
  constexpr float k = 8388736.f;
  return make_float4(__uint_as_float(__byte_perm(x, 0x4b000000u, 0x7440)) - k,
                     __uint_as_float(__byte_perm(x, 0x4b000000u, 0x7441)) - k,
                     __uint_as_float(__byte_perm(x, 0x4b000000u, 0x7442)) - k,
                     __uint_as_float(__byte_perm(x, 0x4b000000u, 0x7443)) - k);
}

// What the rows are: of a cache's pages, of a prompt, or of pages with sums as results.
enum { CACHE = 0, PROMPT_ROWS = 1, PARTS = 2 };

template <int D, bool I8, int NT, int TR, int MODE>
__global__ void __launch_bounds__(NT, 1)
    attend_simt_kernel(const __grid_constant__ AttendJob A, const __grid_constant__ AttendPlan P) {
  using SM = Simt<D, NT, TR>;
  constexpr int BK = SM::BK, NK = SM::NK;
  constexpr bool PROMPT = MODE == PROMPT_ROWS;
  extern __shared__ __align__(16) unsigned char smraw[];
  typename SM::Smem& sm = *reinterpret_cast<typename SM::Smem*>(smraw);
  cache_start();
  const CacheJob& J = A.c;
  const int tid = threadIdx.x, lane = tid % 32, tx = tid % 16, ty = tid / 16;
  const AttendSpan sp = attend_span(A, P, &sm.scan);
  int u = sp.unit;
  int64_t before = sp.before;
  for (int64_t at = sp.begin; at < sp.end;) {
    const AttendUnit U = attend_unit(A, P, sm.scan.lengths(A.c), u);
    const int64_t last = before + U.cost;
    if (last <= at) {
      before = last;
      ++u;
      continue;
    }
    const int64_t stop = min(sp.end, last);
    int s0, s1;
    attend_pieces(U, at, stop, before, s0, s1);
    if (s0 >= s1) {                                    // the unit's start alone
      at = stop;
      continue;
    }
    const int32_t* table = PROMPT ? nullptr : cache_table(J, (size_t)U.b * J.Hkv + U.h);

    for (int i = tid; i < SM::RT * (D / 4); i += NT) {
      const int r = i / (D / 4), d0 = i % (D / 4) * 4;
      uint4 w = make_uint4(0, 0, 0, 0);
      if (r < U.rows) {
        const int tok = J.by_r(U.row0 + r), j = U.row0 + r - tok * J.r;
        w = load_plain16(A.q + ((size_t)(J.off[U.b] + tok) * J.stride + (size_t)(U.h * J.r + j) * D + d0) * 4, A.qvec);
      }
      *reinterpret_cast<uint4*>(&sm.q[r][d0]) = w;
    }
    float m[TR], l[TR];
    int lim[TR];
    uint64_t o[TR][D / 64][2];
#pragma unroll
    for (int i = 0; i < TR; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
      lim[i] = keys_of(A.causal, U.len, U.n, J.by_r(U.row0 + min(ty * TR + i, U.rows - 1)));
#pragma unroll
      for (int c = 0; c < D / 64; ++c) o[i][c][0] = o[i][c][1] = pk2(0.f, 0.f);
    }
    const int least = keys_of(A.causal, U.len, U.n, J.by_r(U.row0));

    // A thread brings 16 bytes of every (16 * NT / row bytes)-th key.
    constexpr int ROWB = I8 ? D : 4 * D, LPR = ROWB / 16, STEP = NT / LPR;   // lanes of a row, keys a round
    constexpr int N = BK / STEP;
    const int lk = tid / LPR, part = tid % LPR;
    uint4 codes[I8 ? N : 1];
    float scale = 0.f;
    // a prompt's rows are K's and V's own, tokens apart
    const int64_t pitch_in = PROMPT ? A.kv_stride * 4 : ROWB;
    auto row_of = [&](int t) {
      if constexpr (PROMPT) return t < U.keys ? J.off[U.b] + t : -1;
      return t < U.keys ? page_row(table[t >> J.page_shift], J.n_pages, J.page_shift, t) : -1;
    };
    auto fetch = [&](int s, const uint8_t* pages, const float* scales, float* dst, int pitch) {
      const uint8_t* from = nullptr;                   // the row of key `lk` of its 16 keys, null without one
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int key = lk + i * STEP, t = s * BK + key;
        if (i * STEP % 16 == 0) {
          const int64_t row = s < s1 ? row_of(t) : -1;
          from = row < 0 ? nullptr : pages + row * pitch_in + part * 16 + (PROMPT ? U.h * ROWB : 0);
        }
        const bool in = from && t < U.keys;
        const uint8_t* src = in ? from + i * STEP % 16 * pitch_in : pages;
        if constexpr (I8) codes[i] = in ? *reinterpret_cast<const uint4*>(src) : make_uint4(0, 0, 0, 0);
        else copy16(dst + key * pitch + part * 4, src, in);
      }
      if constexpr (I8) {
        if (tid < BK) {
          const int row = s < s1 ? row_of(s * BK + tid) : -1;
          scale = row < 0 ? 0.f : scales[row];
        }
      } else {
        copies_commit();
      }
    };
    auto arrive = [&](float* dst, int pitch, float* scales, float by) {   // what fetch() asked for
      if constexpr (I8) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          // Neighbours begin at other quarters of their 16 values: no bank conflicts.
          const int turn = part / 2 % 4;
          uint32_t x[4] = {codes[i].x, codes[i].y, codes[i].z, codes[i].w};
          if (turn & 1) {
            const uint32_t y = x[0];
            x[0] = x[1], x[1] = x[2], x[2] = x[3], x[3] = y;
          }
          if (turn & 2) {
            const uint32_t y = x[0], z = x[1];
            x[0] = x[2], x[1] = x[3], x[2] = y, x[3] = z;
          }
          float4* to = reinterpret_cast<float4*>(dst + (lk + i * STEP) * pitch + part * 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) to[(e + turn) % 4] = codes4(x[e]);
        }
        if (tid < BK) scales[tid] = scale * by;
      } else {
        copies_wait();
      }
    };
    float* const kt = &sm.k[0][0];
    float* const vt = &sm.v[0][0];
    fetch(s0, J.kp, J.ks, kt, SM::QS);
    for (int s = s0; s < s1; ++s) {
      const int k0 = s * BK;
      arrive(kt, SM::QS, sm.ks, A.alpha);
      // the pages of the tile's 16-key blocks
      const bool none = lane < NK && k0 + 16 * lane < U.keys && row_of(k0 + 16 * lane) < 0;
      const uint32_t gone = __ballot_sync(0xffffffffu, none);
      if (gone && tid == 0) set_status(J.status, kStatusBadPage);
      __syncthreads();                                 // K is there; the last tile's V is done with
      fetch(s, J.vp, J.vs, vt, D);

      uint64_t x2[TR][NK];
#pragma unroll
      for (int i = 0; i < TR; ++i)
#pragma unroll
        for (int j = 0; j < NK; ++j) x2[i][j] = pk2(0.f, 0.f);
      const uint32_t qa = smem_u32(&sm.q[ty * TR][0]), ka = smem_u32(&sm.k[tx][0]);
#pragma unroll 2
      for (int d = 0; d < D; d += 4) {
        uint64_t kk[NK][2];
#pragma unroll
        for (int j = 0; j < NK; ++j) lds_2x64(ka + (16 * j * SM::QS + d) * 4, kk[j][0], kk[j][1]);
#pragma unroll
        for (int i = 0; i < TR; ++i) {
          uint64_t q0, q1;
          lds_2x64(qa + (i * SM::QS + d) * 4, q0, q1);
#pragma unroll
          for (int j = 0; j < NK; ++j) x2[i][j] = ffma2(q1, kk[j][1], ffma2(q0, kk[j][0], x2[i][j]));
        }
      }
      const bool masked = k0 + BK > least || gone;
      float x[TR][NK];
      bool raise = false;
#pragma unroll
      for (int i = 0; i < TR; ++i)
#pragma unroll
        for (int j = 0; j < NK; ++j) {
          float a, b;
          upk2(x2[i][j], a, b);
          x[i][j] = (a + b) * (I8 ? sm.ks[tx + 16 * j] : A.alpha);
          if (masked && (k0 + tx + 16 * j >= lim[i] || ((gone >> j) & 1u))) x[i][j] = -INFINITY;
          raise |= x[i][j] > m[i] + kRaise;
        }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int i = 0; i < TR; ++i) {
          float top = m[i];
#pragma unroll
          for (int j = 0; j < NK; ++j) top = fmaxf(top, x[i][j]);
#pragma unroll
          for (int z = 1; z < 16; z <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, z));
          const float f = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - top);
          m[i] = top;
          l[i] *= f;
#pragma unroll
          for (int c = 0; c < D / 64; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float a, b;
              upk2(o[i][c][e], a, b);
              o[i][c][e] = pk2(a * f, b * f);
            }
        }
      }
#pragma unroll
      for (int i = 0; i < TR; ++i)
#pragma unroll
        for (int j = 0; j < NK; ++j) {
          x[i][j] = fast_exp2(x[i][j] - (m[i] == -INFINITY ? 0.f : m[i]));
          l[i] += x[i][j];
        }
      arrive(vt, D, sm.vs, 1.f);
      __syncthreads();                                 // V is there, K is done with
      fetch(s + 1, J.kp, J.ks, kt, SM::QS);
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        const int key = tx + 16 * j;
        const float by = I8 ? sm.vs[key] : 1.f;
#pragma unroll
        for (int i = 0; i < TR; ++i) {
          // below zero: a key that the row does not attend to
          const bool hidden = masked && (k0 + key >= lim[i] || ((gone >> j) & 1u));
          sm.p[key][ty * TR + i] = hidden ? -1.f : I8 ? x[i][j] * by : x[i][j];
        }
      }
      __syncwarp();
      const uint32_t va = smem_u32(&sm.v[0][tx * 4]);
      const float* pp = &sm.p[0][ty * TR];
      auto add = [&](int key, auto mask) {
        uint64_t vv[D / 64][2];
#pragma unroll
        for (int c = 0; c < D / 64; ++c) lds_2x64(va + (key * D + 64 * c) * 4, vv[c][0], vv[c][1]);
        float ww[TR];
        using Some = std::conditional_t<TR == 2, float2, float4>;
#pragma unroll
        for (int i = 0; i < TR; i += sizeof(Some) / 4)
          *reinterpret_cast<Some*>(ww + i) = *reinterpret_cast<const Some*>(pp + key * SM::PS + i);
#pragma unroll
        for (int i = 0; i < TR; ++i) {
          const float w = ww[i];
          if (decltype(mask)::value && w < 0.f) continue;
          const uint64_t w2 = pk2(w, w);
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            o[i][c][0] = ffma2(w2, vv[c][0], o[i][c][0]);
            o[i][c][1] = ffma2(w2, vv[c][1], o[i][c][1]);
          }
        }
      };
      const int end = min(U.keys - k0, BK);
      if (!masked) {
#pragma unroll 4
        for (int key = 0; key < BK; ++key) add(key, std::false_type());
      } else {
        // a zero weight times a value that is not finite would be a NaN
#pragma unroll 1
        for (int key = 0; key < end; ++key) add(key, std::true_type());
      }
      __syncwarp();
    }
    if constexpr (!I8) copies_wait();                  // the fetch behind the last tile copied zeros

    const bool whole = s0 == 0 && s1 == U.pieces;
    const size_t slot = (size_t)attend_slot(blockIdx.x, sp.begin, before) * P.rows;
#pragma unroll
    for (int i = 0; i < TR; ++i) {
      float z = l[i];
#pragma unroll
      for (int e = 1; e < 16; e <<= 1) z += __shfl_xor_sync(0xffffffffu, z, e);
      const int r = ty * TR + i;
      if (r < U.rows) {
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          const int d0 = 64 * c + 4 * tx;
          float4 a;
          upk2(o[i][c][0], a.x, a.y);
          upk2(o[i][c][1], a.z, a.w);
          if (whole) {
            attend_write<float, D, MODE == PARTS>(A, U.b, U.h, U.row0 + r, d0, a, m[i], z);
          } else {
            *reinterpret_cast<float4*>(P.po + (slot + r) * D + d0) = a;
            if (d0 == 0) P.pml[slot + r] = make_float2(m[i], z);
          }
        }
      }
    }
    __syncthreads();
    at = stop;
    if (stop == last) {
      before = last;
      ++u;
    }
  }
}

template <int D, bool I8, int NT, int TR, int MODE>
cudaError_t launch(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  constexpr int bytes = (int)sizeof(typename Simt<D, NT, TR>::Smem);
  const auto kernel = attend_simt_kernel<D, I8, NT, TR, MODE>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != cudaSuccess) return e;
  return launch_kernel(kernel, dim3(P.workers), NT, bytes, st, true, 0, A, P);
}

template <int D, bool I8, int MODE>
cudaError_t launch_rows(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  if (P.rows <= 8) return launch<D, I8, 64, 2, MODE>(A, P, st);
  if (P.rows <= 16) return launch<D, I8, 128, 2, MODE>(A, P, st);
  return launch<D, I8, 256, 8, MODE>(A, P, st);
}

template <int MODE>
cudaError_t launch_pages(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  if (A.c.d == 128) return A.c.i8 ? launch_rows<128, true, MODE>(A, P, st) : launch_rows<128, false, MODE>(A, P, st);
  return A.c.i8 ? launch_rows<64, true, MODE>(A, P, st) : launch_rows<64, false, MODE>(A, P, st);
}

}  // namespace

cudaError_t launch_prompt_simt(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  return A.c.d == 128 ? launch<128, false, 256, 8, PROMPT_ROWS>(A, P, st)
                      : launch<64, false, 256, 8, PROMPT_ROWS>(A, P, st);
}

cudaError_t launch_attend_simt(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  return A.part ? launch_pages<PARTS>(A, P, st) : launch_pages<CACHE>(A, P, st);
}

}  // namespace mmshift
