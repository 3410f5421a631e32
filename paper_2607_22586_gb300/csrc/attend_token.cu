// Attention of few query rows (up to 16 of a request and KV head: single tokens
// under grouped heads, a few drafted tokens) over bfloat16 or 8-bit pages.
//
// Bound by the bytes of K and V, which pass once from global memory to the
// registers of the warp that uses them: no shared memory, no barrier in
// the loop. Each warp takes pieces of KEYS keys of its own and keeps its own
// running maximum, sums and output. Both products are m16n8k16 MMAs with
// the keys (and then the dimensions) as M and the query rows as N, so eight
// rows cost one column block and no product is spent on padding beyond that:
//   S^T [keys x rows] = K Q^T,   O^T [dims x rows] += V^T P^T.
// An MMA sums over its k index in any order, and the order of output
// dimensions is free too, so both are chosen such that a lane's fragment is 16
// (or 8) consecutive bytes of a row: lane (g, c) holds key g's dimensions of
// chunk c for S, and, for O, the keys 2c, 2c + 1, 2c + 8, 2c + 9 of dimension
// chunk g, whose pairs of keys one byte permutation brings together. An 8-bit
// code x becomes bfloat16 without rounding: with u = x & 127, 128 + u is
// the pattern 0x4300 | u, and x = (128 + u) - (128 or, for a negative x, 256). K's
// scale goes to the logit and V's into the weight, before it is rounded.
//
// The maximum is only raised when a logit passes it by 8 (base 2), so the common
// step has one vote and no reduction: weights then stay below 2^8.
#include "attend.cuh"

namespace mmshift {
namespace {

constexpr int NT = 128, NW = NT / 32;
constexpr float kRaise = 8.f;

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The transpose of an 8 x 8 matrix of 16-bit values, two of a row in each lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Two codes, in the low bytes of t's halves, as bfloat16.
__device__ __forceinline__ uint32_t codes_bf16(uint32_t t) {
  const uint32_t a = (t & 0x007f007fu) | 0x43004300u, c = (t & 0x00800080u) | 0x43004300u;
  uint32_t x;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(x) : "r"(a), "r"(c));
  return x;
}

__device__ __forceinline__ bool not_finite2(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

__device__ __forceinline__ uint4 load_stream(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load_stream8(const uint8_t* p) {
  uint2 v;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

// NQ: blocks of eight query rows.
template <int D, bool I8, int NQ>
struct Token {
  static constexpr int ROWB = I8 ? D : 2 * D;
  static constexpr int NB = 256 / ROWB;        // 16-key blocks of a piece: 4 KB of K and of V
  static constexpr int KEYS = 16 * NB;
  static constexpr int KC = ROWB / 64;         // 16-byte chunks of a key per lane
  static constexpr int VW = ROWB / 32;         // words of a value row per lane
  static constexpr int KS = D / 16;            // k steps of S
  static constexpr int MT = D / 16;            // dimension blocks of O
  static constexpr int SROW = D + 4;           // floats between rows in shared memory

  struct alignas(16) Smem {
    float o[NW][8 * NQ][SROW];
    float2 ml[NW][8 * NQ];
    AttendScan<NT> scan;
  };

  // 16 words of K and V rows of a block each: k[half][.] is key g + 8 * half,
  // v[.][.] the keys 2c, 2c + 1, 2c + 8, 2c + 9.
  struct KBlock { uint32_t w[2][4 * KC]; float s[2]; };
  struct VBlock { uint32_t w[4][VW]; float s[2]; };

  static __device__ __forceinline__ void load_k(const CacheJob& J, KBlock& x, int row, int t, int end, int g, int c) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const bool in = row >= 0 && t + 8 * hf + g < end;
      const uint8_t* p = J.kp + ((size_t)row + 8 * hf + g) * ROWB + c * 16;
#pragma unroll
      for (int i = 0; i < KC; ++i) {
        const uint4 v = in ? load_stream(p + i * 64) : make_uint4(0, 0, 0, 0);
        x.w[hf][4 * i] = v.x;
        x.w[hf][4 * i + 1] = v.y;
        x.w[hf][4 * i + 2] = v.z;
        x.w[hf][4 * i + 3] = v.w;
      }
      if constexpr (I8) x.s[hf] = in ? J.ks[(size_t)row + 8 * hf + g] : 0.f;
    }
  }

  static __device__ __forceinline__ void load_v(const CacheJob& J, VBlock& x, int row, int t, int end, int g, int c) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int key = 2 * c + (k & 1) + 8 * (k >> 1);
      const bool in = row >= 0 && t + key < end;
      if constexpr (VW >= 4) {
        const uint8_t* p = J.vp + ((size_t)row + key) * ROWB + g * 16;
#pragma unroll
        for (int i = 0; i < VW / 4; ++i) {
          const uint4 v = in ? load_stream(p + i * 128) : make_uint4(0, 0, 0, 0);
          x.w[k][4 * i] = v.x;
          x.w[k][4 * i + 1] = v.y;
          x.w[k][4 * i + 2] = v.z;
          x.w[k][4 * i + 3] = v.w;
        }
      } else {
        const uint2 v = in ? load_stream8(J.vp + ((size_t)row + key) * ROWB + g * 8) : make_uint2(0, 0);
        x.w[k][0] = v.x;
        x.w[k][1] = v.y;
      }
    }
    if constexpr (I8) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) x.s[hf] = row >= 0 && t + 8 * hf + g < end ? J.vs[(size_t)row + 8 * hf + g] : 0.f;
    }
  }

  // A fragments of k step `s` of S.
  static __device__ __forceinline__ void k_frag(const KBlock& x, int s, uint32_t (&a)[4]) {
    if constexpr (!I8) {
      a[0] = x.w[0][2 * s];
      a[1] = x.w[1][2 * s];
      a[2] = x.w[0][2 * s + 1];
      a[3] = x.w[1][2 * s + 1];
    } else {
      a[0] = codes_bf16(__byte_perm(x.w[0][s], 0, 0x1100));
      a[1] = codes_bf16(__byte_perm(x.w[1][s], 0, 0x1100));
      a[2] = codes_bf16(__byte_perm(x.w[0][s], 0, 0x3322));
      a[3] = codes_bf16(__byte_perm(x.w[1][s], 0, 0x3322));
    }
  }

  // A fragments of dimension block m of O^T: its rows g and g + 8 are two
  // neighbouring dimensions of chunk g.
  static __device__ __forceinline__ void v_frag(const VBlock& x, int m, uint32_t (&a)[4]) {
    if constexpr (!I8) {
      a[0] = __byte_perm(x.w[0][m], x.w[1][m], 0x5410);
      a[1] = __byte_perm(x.w[0][m], x.w[1][m], 0x7632);
      a[2] = __byte_perm(x.w[2][m], x.w[3][m], 0x5410);
      a[3] = __byte_perm(x.w[2][m], x.w[3][m], 0x7632);
    } else if (m % 2 == 0) {
      a[0] = codes_bf16(__byte_perm(x.w[0][m / 2], x.w[1][m / 2], 0x4400));
      a[1] = codes_bf16(__byte_perm(x.w[0][m / 2], x.w[1][m / 2], 0x5511));
      a[2] = codes_bf16(__byte_perm(x.w[2][m / 2], x.w[3][m / 2], 0x4400));
      a[3] = codes_bf16(__byte_perm(x.w[2][m / 2], x.w[3][m / 2], 0x5511));
    } else {
      a[0] = codes_bf16(__byte_perm(x.w[0][m / 2], x.w[1][m / 2], 0x6622));
      a[1] = codes_bf16(__byte_perm(x.w[0][m / 2], x.w[1][m / 2], 0x7733));
      a[2] = codes_bf16(__byte_perm(x.w[2][m / 2], x.w[3][m / 2], 0x6622));
      a[3] = codes_bf16(__byte_perm(x.w[2][m / 2], x.w[3][m / 2], 0x7733));
    }
  }

  // The first of the two dimensions of block m in lanes of chunk g.
  static __device__ __forceinline__ int dim_of(int m, int g) {
    if constexpr (!I8) return (m / 4) * 64 + g * 8 + (m % 4) * 2;
    else return g * (D / 8) + 2 * m;
  }
};

template <int D, bool I8, int NQ>
__global__ void __launch_bounds__(NT, NQ == 1 ? 4 : 3) attend_token_kernel(const __grid_constant__ AttendJob A,
                                                                           const __grid_constant__ AttendPlan P) {
  using T = Token<D, I8, NQ>;
  __shared__ typename T::Smem sm;
  dependent_start();
  const CacheJob& J = A.c;
  const int lane = threadIdx.x % 32, w = threadIdx.x / 32, g = lane / 4, c = lane % 4;
  const AttendSpan sp = attend_span<NT>(A, P, &sm.scan, [] { __syncthreads(); });
  int u = sp.unit;
  int64_t before = sp.before;
  for (int64_t at = sp.begin; at < sp.end;) {
    const AttendUnit U = attend_unit(A, P, u);
    const int64_t last = before + U.pieces;
    if (last <= at) {                                  // a unit without pieces
      before = last;
      ++u;
      continue;
    }
    const int64_t stop = min(sp.end, last);
    const int s0 = (int)(at - before), s1 = (int)(stop - before);
    const int32_t* table = J.table + ((size_t)U.b * J.Hkv + U.h) * J.max_pages;

    // query rows as B fragments: row 8 * nq + g
    uint32_t q[NQ][2 * T::KS];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int row = 8 * nq + g;
      const bool in = row < U.rows;
      const int tok = in ? row / J.r : 0, j = in ? row - tok * J.r : 0;
      const uint8_t* p = A.q + ((size_t)(J.off[U.b] + tok) * J.stride + (size_t)(U.h * J.r + j) * D) * 2;
#pragma unroll
      for (int i = 0; i < 2 * T::KS / 4; ++i) {
        // words of k steps 2i, 2i + 1: dimensions 8c.. of each 32 (bfloat16 pages), 16c.. of each 64 (codes)
        const int d0 = I8 ? (i / 2) * 64 + c * 16 + (i % 2) * 8 : i * 32 + c * 8;
        const uint4 v = in ? load_plain16(p + d0 * 2, A.qvec) : make_uint4(0, 0, 0, 0);
        q[nq][4 * i] = v.x;
        q[nq][4 * i + 1] = v.y;
        q[nq][4 * i + 2] = v.z;
        q[nq][4 * i + 3] = v.w;
      }
    }
    // rows 8 * nq + 2c and + 1 as columns of the products
    float m[NQ][2], l[NQ][2], o[NQ][T::MT][4];
    int lim[NQ][2];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[nq][e] = -INFINITY;
        l[nq][e] = 0.f;
        lim[nq][e] = keys_of(A.causal, U.len, U.n, min(8 * nq + 2 * c + e, U.rows - 1) / J.r);
#pragma unroll
        for (int mt = 0; mt < T::MT; ++mt) o[nq][mt][e] = o[nq][mt][2 + e] = 0.f;
      }
    const int least = keys_of(A.causal, U.len, U.n, 0);   // keys that every row attends to

    // row of the pool of each 16-key block, -1 behind the end and without a page
    auto rows_of = [&](int s, int (&row)[T::NB]) {
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) {
        const int t = s * T::KEYS + 16 * nb;
        row[nb] = s < s1 && t < U.keys ? page_row(table[t >> J.page_shift], J.n_pages, J.page_shift, t) : -1;
      }
    };
    typename T::KBlock kb[T::NB];
    typename T::VBlock vb[T::NB];
    int row[T::NB], next[T::NB];
    int s = s0 + w;
    rows_of(s, row);
    rows_of(s + NW, next);
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb) T::load_k(J, kb[nb], row[nb], s * T::KEYS + 16 * nb, U.keys, g, c);
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb) T::load_v(J, vb[nb], row[nb], s * T::KEYS + 16 * nb, U.keys, g, c);

    for (; s < s1; s += NW) {
      const int t0 = s * T::KEYS;
      float x[NQ][T::NB][4];                           // keys g, g | g + 8, g + 8; rows 2c, 2c + 1
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[nq][nb][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < T::KS; ++ks) {
          uint32_t a[4];
          T::k_frag(kb[nb], ks, a);
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq) mma16816(x[nq][nb], a[0], a[1], a[2], a[3], q[nq][2 * ks], q[nq][2 * ks + 1]);
        }
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[nq][nb][i] *= I8 ? A.alpha * kb[nb].s[i / 2] : A.alpha;
      }
      const int tn = t0 + NW * T::KEYS;
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) T::load_k(J, kb[nb], next[nb], tn + 16 * nb, U.keys, g, c);

      bool gone = false;
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) gone |= row[nb] < 0 && t0 + 16 * nb < U.keys;
      const bool masked = t0 + T::KEYS > least || gone;
      if (masked) {
        if (gone && lane == 0) set_status(J.status, kStatusBadPage);
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (row[nb] < 0 || t0 + 16 * nb + 8 * (i / 2) + g >= lim[nq][i % 2]) x[nq][nb][i] = -INFINITY;
      }
      bool raise = false;
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
          for (int i = 0; i < 4; ++i) raise |= x[nq][nb][i] > m[nq][i % 2] + kRaise;
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = m[nq][e];
#pragma unroll
            for (int nb = 0; nb < T::NB; ++nb) top = fmaxf(top, fmaxf(x[nq][nb][e], x[nq][nb][2 + e]));
#pragma unroll
            for (int z = 4; z < 32; z <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, z));
            const float f = m[nq][e] == -INFINITY ? 0.f : fast_exp2(m[nq][e] - top);
            m[nq][e] = top;
            l[nq][e] *= f;
#pragma unroll
            for (int mt = 0; mt < T::MT; ++mt) {
              o[nq][mt][e] *= f;
              o[nq][mt][2 + e] *= f;
            }
          }
      }
      uint32_t p[NQ][T::NB][2];
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
        const float m0 = m[nq][0] == -INFINITY ? 0.f : m[nq][0], m1 = m[nq][1] == -INFINITY ? 0.f : m[nq][1];
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb) {
          float e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            e[i] = fast_exp2(x[nq][nb][i] - (i % 2 ? m1 : m0));
            l[nq][i % 2] += e[i];
          }
          if constexpr (I8) {
            // a key that is masked has no part in the result, whatever its scale
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = masked && x[nq][nb][i] == -INFINITY ? 0.f : e[i] * vb[nb].s[i / 2];
          }
          p[nq][nb][0] = transpose8(pack_bf16(e[0], e[1]));
          p[nq][nb][1] = transpose8(pack_bf16(e[2], e[3]));
        }
      }
      bool plain = true;
      if constexpr (!I8) {
        // A zero weight times a value that is not finite is a NaN. Where a tile has
        // such values behind some row's last key, the keys are multiplied one by one
        // and a row takes only those that it attends to.
        if (masked) {
          bool odd = false;
#pragma unroll
          for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int i = 0; i < T::VW; ++i) odd |= not_finite2(vb[nb].w[k][i]);
          plain = !__any_sync(0xffffffffu, odd);
        }
      }
      if (plain) {
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
          for (int mt = 0; mt < T::MT; ++mt) {
            uint32_t a[4];
            T::v_frag(vb[nb], mt, a);
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) mma16816(o[nq][mt], a[0], a[1], a[2], a[3], p[nq][nb][0], p[nq][nb][1]);
          }
      } else {
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll 1
          for (int k = 0; k < 16; ++k) {
            const uint32_t half = (k & 7) >> 1 == c ? (k & 1 ? 0xffff0000u : 0xffffu) : 0u;
            const uint32_t lo = k < 8 ? half : 0u, hi = k < 8 ? 0u : half;
#pragma unroll
            for (int mt = 0; mt < T::MT; ++mt) {
              uint32_t a[4];
              T::v_frag(vb[nb], mt, a);
#pragma unroll
              for (int nq = 0; nq < NQ; ++nq) {
                float d[4] = {};
                mma16816(d, a[0] & lo, a[1] & lo, a[2] & hi, a[3] & hi, p[nq][nb][0], p[nq][nb][1]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  if (t0 + 16 * nb + k < lim[nq][i % 2]) o[nq][mt][i] += d[i];
              }
            }
          }
      }
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) T::load_v(J, vb[nb], next[nb], tn + 16 * nb, U.keys, g, c);
#pragma unroll
      for (int nb = 0; nb < T::NB; ++nb) row[nb] = next[nb];
      rows_of(s + 2 * NW, next);
    }

    // the warps' sums together
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float z = l[nq][e];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) z += __shfl_xor_sync(0xffffffffu, z, d);
        const int r = 8 * nq + 2 * c + e;
        if (g == 0) sm.ml[w][r] = make_float2(m[nq][e], z);
#pragma unroll
        for (int mt = 0; mt < T::MT; ++mt)
          *reinterpret_cast<float2*>(&sm.o[w][r][T::dim_of(mt, g)]) = make_float2(o[nq][mt][e], o[nq][mt][2 + e]);
      }
    __syncthreads();
    const bool whole = s0 == 0 && s1 == U.pieces;
    const size_t slot = (size_t)attend_slot(blockIdx.x, sp.begin, before) * P.rows;
    for (int i = threadIdx.x; i < U.rows * (D / 4); i += NT) {
      const int r = i / (D / 4), d0 = i % (D / 4) * 4;
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < NW; ++k) top = fmaxf(top, sm.ml[k][r].x);
      float z = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        const float2 ml = sm.ml[k][r];
        // a warp without a maximum has zeros, or NaN that have to stay
        const float f = ml.x == -INFINITY ? 1.f : fast_exp2(ml.x - top);
        const float4 v = *reinterpret_cast<const float4*>(&sm.o[k][r][d0]);
        z += ml.y * f;
        acc.x += v.x * f;
        acc.y += v.y * f;
        acc.z += v.z * f;
        acc.w += v.w * f;
      }
      if (whole) {
        attend_write<__nv_bfloat16, D>(A, U.b, U.h, r, d0, acc, top, z);
      } else {
        *reinterpret_cast<float4*>(P.po + (slot + r) * D + d0) = acc;
        if (d0 == 0) P.pml[slot + r] = make_float2(top, z);
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

}  // namespace

cudaError_t launch_attend_token(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  auto go = [&](auto kernel) { return launch_kernel(kernel, dim3(P.workers), NT, 0, st, true, 0, A, P); };
  const CacheJob& J = A.c;
  if (P.rows <= 8) {
    if (J.d == 128) return J.i8 ? go(attend_token_kernel<128, true, 1>) : go(attend_token_kernel<128, false, 1>);
    return J.i8 ? go(attend_token_kernel<64, true, 1>) : go(attend_token_kernel<64, false, 1>);
  }
  if (J.d == 128) return J.i8 ? go(attend_token_kernel<128, true, 2>) : go(attend_token_kernel<128, false, 2>);
  return J.i8 ? go(attend_token_kernel<64, true, 2>) : go(attend_token_kernel<64, false, 2>);
}

}  // namespace mmshift
