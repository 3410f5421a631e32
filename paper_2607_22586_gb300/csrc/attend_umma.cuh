// What the tensor-core attention kernels share: products from tensor memory, its loads and
// stores, values that are not finite, and a CTA's runs of keys.
#pragma once

#include "attend.cuh"
#include "umma.cuh"

namespace mmshift {

constexpr int BQ = 128, BK = 128;      // rows of a block, keys of a tile
constexpr float kRaise = 8.f;          // a row's maximum is raised when a logit passes it by this (base 2)

namespace umma {

__device__ __forceinline__ void mma_p(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                      uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// B operand whose rows are keys: 64 columns of 8 keys a 1024-byte swizzled atom,
// groups of 8 keys 1024 bytes apart, the next 64 columns `half` bytes on.
__device__ __forceinline__ uint64_t sdesc_mn_sw128(uint32_t saddr, uint32_t half) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(half >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}

// 32 columns of the warp's 32 lanes; what was read may be used after ld_wait on it.
__device__ __forceinline__ void ld32(uint32_t taddr, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
        "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
        "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr));
}
__device__ __forceinline__ void pin32(float* v) {
  asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                    "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]),
                    "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]),
                    "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]),
                    "+f"(v[29]), "+f"(v[30]), "+f"(v[31]));
}
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ bool not_finite2(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ uint32_t finite2(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}

// The largest of N values (a NaN is passed over), N a multiple of 8.
template <int N>
__device__ __forceinline__ float max_of(const float* v) {
  float t[4] = {fmaxf(v[0], v[4]), fmaxf(v[1], v[5]), fmaxf(v[2], v[6]), fmaxf(v[3], v[7])};
#pragma unroll
  for (int i = 8; i < N; i += 8)
#pragma unroll
    for (int c = 0; c < 4; ++c) t[c] = fmaxf(t[c], fmaxf(v[i + c], v[i + 4 + c]));
  return fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
}

// A value that is the same in all lanes, so that the compiler knows that it is.
__device__ __forceinline__ int uniform(int x) { return (int)__reduce_max_sync(0xffffffffu, (unsigned)x); }

// A converged warp's wait, as umma.cuh's, without a vote a poll (2 % of a long chunk).
__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity, volatile int* abort) {
  const bool ok = mbar_try_wait_fast(bar, parity) || mbar_wait(bar, parity, abort);
  return __all_sync(0xffffffffu, ok);
}

}  // namespace umma

// A run: consecutive key tiles [s0, s1) of a unit that the CTA works on together.
struct Run {
  AttendUnit U;
  int64_t before;        // costs before the unit
  int s0, s1;
  bool two;              // the second block has rows
  int x;                 // else: the block that has them, each in turn
  __device__ __forceinline__ bool has(int b) const { return two || b == x; }
  __device__ __forceinline__ int first_row(int b) const { return two ? b * BQ : 0; }   // of block b in the tile
};

// A role's walk over the CTA's runs. A warp works the first ones out for all roles, a
// lane a unit; a role itself those behind them (units of few keys).
struct Walk {
  int runs, k, unit;     // runs so far, those of the list; behind it, the next unit and the costs before it
  int64_t before;
};
template <int RUNS>
struct RunList {
  Run run[RUNS];
  Walk rest;
  int n;
};

__device__ __forceinline__ Run run_of(const AttendSpan& sp, const AttendUnit& U, int64_t before) {
  Run R;
  R.U = U;
  R.before = before;
  attend_pieces(U, sp.begin, sp.end, before, R.s0, R.s1);
  R.two = U.rows > BQ;
  return R;
}

// By a whole warp: the first runs of the CTA.
template <int RUNS>
__device__ __forceinline__ void list_runs(const AttendJob& A, const AttendPlan& P, const AttendSpan& sp, int lane,
                                          RunList<RUNS>* list) {
  const int u = sp.unit + lane;
  const bool in = sp.begin < sp.end && lane < RUNS && u < P.uoff[A.c.B];
  AttendUnit U;
  U.pieces = U.extra = U.cost = 0;
  if (in) U = attend_unit(A, P, nullptr, u);
  int64_t x = U.cost;
#pragma unroll
  for (int d = 1; d < RUNS; d <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  const int64_t before = sp.before + x - U.cost;
  const Run R = run_of(sp, U, before);
  const bool mine = in && R.s0 < R.s1;
  const unsigned all = __ballot_sync(0xffffffffu, mine);
  if (mine) list->run[__popc(all & ((1u << lane) - 1u))] = R;
  if (lane == RUNS - 1) {                              // where the walk goes on
    list->n = __popc(all);
    list->rest = Walk{0, 0, u + 1, in ? sp.before + x : sp.end};
  }
}

template <int RUNS>
__device__ __forceinline__ bool next_run(const AttendJob& A, const AttendPlan& P, const AttendSpan& sp,
                                         const RunList<RUNS>& list, Walk& w, Run& R) {
  bool found = w.k < list.n;
  if (found) {
    R = list.run[w.k++];
  } else {
    if (w.k == list.n) {
      w.k = RUNS + 1;
      w.unit = list.rest.unit;
      w.before = list.rest.before;
    }
    while (!found && w.before < sp.end) {
      const AttendUnit U = attend_unit(A, P, nullptr, w.unit);
      R = run_of(sp, U, w.before);
      w.before += U.cost;
      ++w.unit;
      found = R.s0 < R.s1;
    }
  }
  R.x = w.runs++ & 1;
  return found;
}

}  // namespace mmshift
