// Attention over whole prompts of bfloat16 rows on the 5th-generation tensor cores
// (tcgen05 + TMA + TMEM).
//
// Tiles of 256 query rows (two blocks of 128, a token's heads next to one another) over tiles of
// 128 keys, S = Q K^T and O += P V as in the chunk kernel (attend_umma.cu): S and P in
// tensor memory, one softmax thread a row. Prompts have many tiles of few keys (a prompt of
// 1000 tokens and seven heads a KV head has 28 tiles, of 5 key tiles on average), so a
// run's start and end are other warps' work, and the products go on from run to run:
//   warps 0-7   softmax, a warpgroup a block;
//   warp 8      TMA producer of K and V tiles;
//   warp 9      MMA issuer, one thread: a block's first S of the next run follows its last P V;
//   warps 10-11 load Q of the next blocks into a ring of three places;
//   warps 12-15 clean V where a tile is masked, and take O out: 104 registers a thread.
// The issuer is alone in its warp, and what it asks for is in registers: while the products read
// shared memory at its full rate, an access there takes hundreds of cycles, and the issuer's
// own path is what the tensor cores wait for.
// K's and V's rows are tokens apart: a tile is one box of 128 rows. Rows behind a prompt's last
// are the next prompt's: a zero weight times a NaN there would be a NaN, so in tiles that hold
// keys which some row does not attend to, values that are not finite are set to zero
// for the product and added to the rows that do attend to them at the end.
// Every wait is bounded; a role that gives up ends the CTA as score_umma.cu says.
#include <algorithm>

#include "attend_umma.cuh"

namespace mmshift {
namespace {

using namespace umma;

constexpr int PRODUCER = 8, ISSUER = 9, LOADER = 10, FINISHER = 12;   // first warps of the roles
// Registers a thread of the softmax warpgroups and of the others: in all as many as at the launch.
constexpr int SOFTMAX_REGS = 152, OTHER_REGS = 104;

template <int D>
struct PromptSmem {
  static constexpr int NT = 512;
  static_assert(256 * (SOFTMAX_REGS + OTHER_REGS) <= 512 * 128, "more registers than the launch has");
  static constexpr int HALVES = D / 64;
  static constexpr int HALF = BK * 128;              // 64 columns of 128 rows
  static constexpr int TILE = HALVES * HALF;         // a block of Q, a tile of K or V
  static constexpr int QS = 3;                       // blocks of Q
  static constexpr int STAGES = D == 64 ? 8 : 4;
  // Before the tiles: barriers and what roles tell one another. All of the CTA's shared memory is
  // asked for, and none declared besides, so the tiles' alignment costs nothing.
  struct Head {
    uint64_t full[STAGES], empty[STAGES], q_full[QS], q_empty[QS];
    uint64_t s_ready[2], p_ready[2], o_ready[2], o_free[2], l_ready[2], v_ask, v_clean, drain;
    union {
      AttendScan<NT, 1> scan;          // before the roles begin
      float2 ml[2][BQ];                // a block's rows: maximum (base 2) and sum of weights
    };
    RunList<8> runs;
    uint32_t tbase;
    int abort_flag, odd_flag;
  };
  static constexpr int BYTES = 227 * 1024;
  static_assert((QS + STAGES) * TILE + 3 * 1024 <= BYTES && sizeof(Head) <= 3 * 1024, "shared memory");
  static constexpr uint32_t O_COL = 256, O_STRIDE = D;
};

// Start: everything before in the stream is done, and the next kernel may take its place.
__device__ __forceinline__ void prompt_start() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// The part of a row's sums that comes from values that are not finite, of columns
// [d0, d0 + 32): added with the row's weights, key by key. Rare, so slow.
template <int D>
__device__ __forceinline__ void add_not_finite(const AttendJob& A, const Run& R, int row, int lim, float m, int d0,
                                                   float* o) {
  const CacheJob& J = A.c;
  const int tok = J.by_r(row), j = row - tok * J.r;
  const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(A.q) +
                           (size_t)(J.off[R.U.b] + tok) * J.stride + (size_t)(R.U.h * J.r + j) * D;
  const int first = keys_of(A.causal, R.U.len, R.U.n, J.by_r(R.U.row0));
  for (int t = max(R.s0 * BK, first / BK * BK); t < min(R.s1 * BK, lim); ++t) {
    const size_t at = (size_t)(J.off[R.U.b] + t) * A.kv_stride + (size_t)R.U.h * D;
    const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(J.vp) + at + d0;
    bool any = false;
    for (int i = 0; i < 32; ++i) any |= !isfinite(to_f32(v[i]));
    if (!any) continue;
    const __nv_bfloat16* k = reinterpret_cast<const __nv_bfloat16*>(J.kp) + at;
    float s = 0.f;
    for (int i = 0; i < D; ++i) s = fmaf(to_f32(q[i]), to_f32(k[i]), s);
    const float p = fast_exp2(fmaf(s, A.alpha, -m));
    for (int i = 0; i < 32; ++i) {
      const float x = to_f32(v[i]);
      if (!isfinite(x)) o[i] += p * x;
    }
  }
}

// Key tiles [s0, end) of a run that block b works on: rows in front may see fewer keys than the
// tile's last one. One at least, so that the block has sums.
__device__ __forceinline__ int block_end(const AttendJob& A, const Run& R, int b) {
  const int last = min(R.U.rows, R.first_row(b) + BQ) - 1;
  const int keys = keys_of(A.causal, R.U.len, R.U.n, A.c.by_r(R.U.row0 + last));
  return max(min(R.s1, (keys + BK - 1) / BK), R.s0 + 1);
}

__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS)); }

// A bounded wait without a call (umma.cuh): a function's registers are not known where a role has
// given some of its own away, or taken more.
__device__ __forceinline__ bool wait_one(uint64_t* bar, uint32_t parity, volatile int* abort) {
#pragma unroll 1
  for (uint32_t i = 0; i < kFastPolls; ++i)
    if (mbar_try_wait_fast(bar, parity)) return true;
#pragma unroll 1
  for (uint32_t i = 0; i < kSpinLimit; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort) return false;
  }
  *abort = 1;
  return false;
}
// By a converged warp, which stays converged.
__device__ __forceinline__ bool wait_all(uint64_t* bar, uint32_t parity, volatile int* abort) {
  return __all_sync(0xffffffffu, wait_one(bar, parity, abort));
}

// A value that is the same in all lanes, where the compiler knows that it is.
__device__ __forceinline__ int uniform(int x) { return (int)__reduce_max_sync(0xffffffffu, (unsigned)x); }

// What the issuer has to know of a run.
struct IssueRun {
  int s0, s1, end0, end1, masked;      // masked: the first tile whose V is cleaned
  int blocks, use;                     // bit b: block b has rows; its Q is use + (blocks == 3 ? b : 0)
};

// 32 bytes of a row at once where the address allows.
__device__ __forceinline__ void store32(uint8_t* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

template <int D>
__global__ void __launch_bounds__(PromptSmem<D>::NT, 1) attend_prompt_kernel(const __grid_constant__ CUtensorMap kmap,
                                                              const __grid_constant__ CUtensorMap vmap,
                                                              const __grid_constant__ AttendJob A,
                                                              const __grid_constant__ AttendPlan P) {
  using SM = PromptSmem<D>;
  extern __shared__ __align__(16) unsigned char smraw[];
  typename SM::Head& hd = *reinterpret_cast<typename SM::Head*>(smraw);
  unsigned char* sm = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smraw) + sizeof(typename SM::Head) + 1023) & ~uintptr_t(1023));
  unsigned char* ring = sm + SM::QS * SM::TILE;
  uint64_t *const full = hd.full, *const empty = hd.empty, *const q_full = hd.q_full, *const q_empty = hd.q_empty;
  uint64_t *const s_ready = hd.s_ready, *const p_ready = hd.p_ready, *const o_ready = hd.o_ready;
  uint64_t *const o_free = hd.o_free, *const l_ready = hd.l_ready;
  auto& runs = hd.runs;
  if (sm + (SM::QS + SM::STAGES) * SM::TILE > smraw + SM::BYTES) {   // the base is not where it always is
    if (threadIdx.x == 0) set_status(A.c.status, kStatusTimeout);
    return;
  }
  // Every role passes all fills of the barriers that it waits for, in order, and none runs ahead of
  // the wait of another by more than one: a parity says which fill is meant.
  volatile int* abort_ = &hd.abort_flag;
  const CacheJob& J = A.c;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

  if (threadIdx.x == 0) {
    hd.abort_flag = hd.odd_flag = 0;
    for (int s = 0; s < SM::STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < SM::QS; ++s) {
      mbar_init(&q_full[s], 2);      // both loaders
      mbar_init(&q_empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_ready[i], 1);
      mbar_init(&p_ready[i], 4);     // a warpgroup's warps
      mbar_init(&o_ready[i], 1);
      mbar_init(&o_free[i], 4);
      mbar_init(&l_ready[i], 4);
    }
    mbar_init(&hd.v_ask, 1);
    mbar_init(&hd.v_clean, 4);
    mbar_init(&hd.drain, 1);
    fence_barrier_init();
    prefetch_tmap(&kmap);
    prefetch_tmap(&vmap);
  }
  if (warp == ISSUER) {
    tmem_alloc(&hd.tbase, 512);
    tmem_relinquish();
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = hd.tbase;
  prompt_start();
  const AttendSpan sp = attend_span(A, P, &hd.scan);
  if (warp == 0) list_runs(A, P, sp, lane, &runs);
  __syncthreads();
  Walk walk = {0, 0, 0, 0};
  Run R;
  // Blocks of Q are used in the order of the runs, a run's first block first: use n lies in
  // place n % QS.
  if (warp == PRODUCER) {
    fewer_registers();
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      ArmedStages armed;
      bool ok = true;
      while (ok && next_run(A, P, sp, runs, walk, R)) {
        const int row0 = J.off[R.U.b], col0 = R.U.h * D;
        for (int s = R.s0; ok && s < R.s1; ++s) {
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            if (!wait_one(&empty[stage], phase ^ 1u, abort_)) { ok = false; break; }
            mbar_expect_tx(&full[stage], SM::TILE);
#pragma unroll
            for (int c = 0; c < SM::HALVES; ++c)
              tma_load_3d(ring + stage * SM::TILE + c * SM::HALF, kv ? &vmap : &kmap, &full[stage], col0 + c * 64,
                          row0 + s * BK, 0);
            armed.arm(stage, phase);
            if (++stage == SM::STAGES) { stage = 0; phase ^= 1u; }
          }
        }
      }
      if (!armed.drain(full)) *abort_ = 1;
    }
    __syncwarp();
  } else if (warp == ISSUER) {
    fewer_registers();
    {
      const uint32_t id_s = idesc_bf16_f32(BQ, BK), id_o = idesc_bf16_f32(BQ, D) | (1u << 16);   // V: MN-major
      const uint64_t qd = sdesc_k_sw128(smem_u32(sm)), kd = sdesc_k_sw128(smem_u32(ring));
      const uint64_t vd = sdesc_mn_sw128(smem_u32(ring), SM::HALF);
      int stage = 0, use = 0;
      uint32_t phase = 0, pp = 0, of = 0, vc = 0;      // of the ring, of block i's barriers (bit i), of v_clean
      bool ok = true, issued = false;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        ok = ok && wait_all(bar, parity & 1u, abort_);
        return ok;
      };
      auto step = [&] {
        if (++stage == SM::STAGES) { stage = 0; phase ^= 1u; }
      };
      auto next = [&](IssueRun& r) {
        if (!__all_sync(0xffffffffu, next_run(A, P, sp, runs, walk, R))) return false;
        r.s0 = uniform(R.s0);
        r.s1 = uniform(R.s1);
        r.end0 = uniform(R.has(0) ? block_end(A, R, 0) : R.s0);
        r.end1 = uniform(R.has(1) ? block_end(A, R, 1) : R.s0);
        r.masked = uniform(keys_of(A.causal, R.U.len, R.U.n, J.by_r(R.U.row0)) / BK);
        r.blocks = uniform(R.two ? 3 : 1 << R.x);
        r.use = use;
        use += r.blocks == 3 ? 2 : 1;
        return true;
      };
      auto commit = [&](uint64_t* bar) {
        if (elect_one()) mma_commit(bar);
        __syncwarp();
      };
      // S of block x, whose Q is in a place, with the K tile of the stage
      auto issue_s = [&](int x, int place) {
        const uint64_t k = kd + (uint64_t)(stage * (SM::TILE >> 4)), q = qd + (uint64_t)(place * (SM::TILE >> 4));
        if (elect_one()) {
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint64_t o = (uint64_t)(((ks / 4) * SM::HALF + (ks % 4) * 32) >> 4);
            mma_bf16(tmem + x * BK, q + o, k + o, id_s, ks > 0 ? 1u : 0u);
          }
          mma_commit(&s_ready[x]);
        }
        __syncwarp();
        issued = true;
      };
      // the first S of a run
      auto first_s = [&](const IssueRun& r, int x) {
        const int n = r.use + (r.blocks == 3 ? x : 0), place = n % SM::QS;
        if (!wait(&q_full[place], (uint32_t)(n / SM::QS))) return;
        fence_after();
        issue_s(x, place);
        if ((x ? r.end1 : r.end0) == r.s0 + 1) commit(&q_empty[place]);
      };
      auto issue_o = [&](int x, int st, bool add) {
        const uint64_t v = vd + (uint64_t)(st * (SM::TILE >> 4));
        if (elect_one()) {
#pragma unroll
          for (int ks = 0; ks < BK / 16; ++ks)
            mma_p(tmem + SM::O_COL + x * SM::O_STRIDE, tmem + x * BK + ks * 8, v + (uint64_t)((ks * 2048) >> 4), id_o,
                  add || ks > 0 ? 1u : 0u);
        }
        __syncwarp();
      };
      IssueRun r, n;
      bool have = next(r);
      if (have && wait(&full[stage], phase)) {
        for (int x = 0; ok && x < 2; ++x)
          if (r.blocks >> x & 1) first_s(r, x);
        commit(&empty[stage]);
        step();
      }
      while (ok && have) {
        const bool more = next(n);
        const int place0 = r.use % SM::QS, place1 = (r.use + 1) % SM::QS;
        for (int s = r.s0; ok && s < r.s1; ++s) {
          // In order: P V of a tile reads P before S of the next tile (of this run or the next) takes
          // its place. While one block's products run, the other's softmax does.
          const int vst = stage;
          const bool last = s + 1 == r.s1;
          bool k_there = false, v_there = s < r.masked;
          if (!wait(&full[vst], phase)) break;
          if (!v_there) {
            if (lane == 0) mbar_arrive(&hd.v_ask);
          }
          step();
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int end = x ? r.end1 : r.end0;
            if (s < end) {
              if (s == r.s0) {                         // the block's last O has been read
                if (!wait(&o_free[x], (of >> x) ^ 1u)) break;
                of ^= 1u << x;
              }
              if (!wait(&p_ready[x], pp >> x)) break;
              pp ^= 1u << x;
              if (!v_there) {
                if (!wait(&hd.v_clean, vc)) break;
                vc ^= 1u;
                v_there = true;
              }
              fence_after();
              issue_o(x, vst, s > r.s0);
              if (s + 1 == end) commit(&o_ready[x]);
            }
            if (x == (s < r.end1 ? 1 : 0)) commit(&empty[vst]);   // the run's last block has had the tile's V
            if (last ? more && (n.blocks >> x & 1) : s + 1 < end) {
              if (!k_there && !wait(&full[stage], phase)) break;
              k_there = true;
              if (last) {
                first_s(n, x);
              } else {
                const int place = x && r.blocks == 3 ? place1 : place0;
                issue_s(x, place);
                if (s + 2 == end) commit(&q_empty[place]);
              }
            }
          }
          if (!ok) break;
          if (!last || more) {
            commit(&empty[stage]);
            step();
          }
        }
        r = n;
        have = more;
      }
      if (issued) {
        commit(&hd.drain);
        if (!mbar_wait_drain(&hd.drain, 0)) *abort_ = 1;
      }
    }
  } else if (warp >= FINISHER) {
    fewer_registers();
    const int fw = warp - FINISHER;
    const uint32_t lanes = (uint32_t)(fw * 32) << 16;
    uint32_t ask = 0, oph = 0;                           // phase of v_ask; bit x: of block x's o_ready
    int stage = 1;                                       // of the next tile's V
    bool ok = true;
    while (ok && next_run(A, P, sp, runs, walk, R)) {
      const AttendUnit& U = R.U;
      const int least = keys_of(A.causal, U.len, U.n, J.by_r(U.row0));   // keys that every row attends to
      for (int s = R.s0; s < R.s1; ++s) {
        const int vs = stage;
        stage = (stage + 2) % SM::STAGES;
        const int k0 = s * BK;
        if (k0 + BK <= least) continue;
        if (!wait_all(&hd.v_ask, ask, abort_)) { ok = false; break; }
        ask ^= 1u;
        unsigned char* vt = ring + vs * SM::TILE;
        constexpr int CH = SM::HALVES * 8;               // 16-byte chunks of a row
        const int i0 = max(least - k0, 0) * CH;
#pragma unroll 4
        for (int i = i0 + fw * 32 + lane; i < BK * CH; i += 128) {
          const int key = i / CH, ch = i % CH;
          uint4* p = reinterpret_cast<uint4*>(vt + (ch / 8) * SM::HALF + key * 128 + (ch % 8) * 16);
          const uint4 w = k0 + key < U.keys ? *p : make_uint4(0, 0, 0, 0);
          const bool bad = not_finite2(w.x) || not_finite2(w.y) || not_finite2(w.z) || not_finite2(w.w);
          if (bad) *reinterpret_cast<volatile int*>(&hd.odd_flag) = 1;
          if (bad || k0 + key >= U.keys) *p = make_uint4(finite2(w.x), finite2(w.y), finite2(w.z), finite2(w.w));
        }
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&hd.v_clean);
      }
      for (int x = 0; ok && x < 2; ++x) {
        if (!R.has(x)) continue;
        const uint32_t ph = oph >> x & 1u;
        if (!wait_all(&l_ready[x], ph, abort_) || !wait_all(&o_ready[x], ph, abort_)) { ok = false; break; }
        oph ^= 1u << x;
        fence_after();
        const int lrow = fw * 32 + lane, brow = R.first_row(x) + lrow, row = U.row0 + brow;
        const bool live = brow < U.rows;
        const int tok = J.by_r(row), j = row - tok * J.r;
        const float2 t = hd.ml[x][lrow];
        const float m = t.x, l = t.y;
        // set by this warp's lanes or those beside it, before they reported a tile clean whose product
        // is in O by now
        const bool fix = *reinterpret_cast<volatile int*>(&hd.odd_flag) != 0;
        const bool whole = R.s0 == 0 && R.s1 == U.pieces;
        const float f = l == 0.f ? 0.f : 1.f / l;
        const int64_t orow = (int64_t)(J.off[U.b] + tok) * J.Hq + U.h * J.r + j;
        const int64_t slot = (int64_t)attend_slot(blockIdx.x, sp.begin, R.before) * P.rows + brow;
        const uint32_t ocol = tmem + lanes + SM::O_COL + x * SM::O_STRIDE;
#pragma unroll 1
        for (int i = 0; i < D; i += 32) {
          float o[32];
          ld32(ocol + i, o);
          tmem_wait_ld();
          pin32(o);
          if (i + 32 == D) {                             // the block's next products may take O's place
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&o_free[x]);
          }
          if (!live) continue;
          if (fix) {
            float y[32];
#pragma unroll
            for (int c = 0; c < 32; ++c) y[c] = o[c];
            add_not_finite<D>(A, R, row, keys_of(A.causal, U.len, U.n, tok), m == -INFINITY ? 0.f : m, i, y);
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] = y[c];
          }
          if (whole) {
            uint32_t w[16];
#pragma unroll
            for (int c = 0; c < 16; ++c) w[c] = l == 0.f ? 0u : pack_bf16(o[2 * c] * f, o[2 * c + 1] * f);
            uint8_t* const to = A.out + (orow * D + i) * 2;
            if (A.ovec == 2) {
              store32(to, w);
              store32(to + 32, w + 8);
            } else {
#pragma unroll
              for (int c = 0; c < 4; ++c)
                store_row16(to + c * 16, make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]), A.ovec);
            }
          } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
              store32(reinterpret_cast<uint8_t*>(P.po + slot * D + i + 8 * c), reinterpret_cast<const uint32_t*>(o + 8 * c));
          }
        }
        if (live) {
          if (!whole) P.pml[slot] = t;
          else if (A.lse) A.lse[orow] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        }
      }
    }
  } else if (warp >= LOADER) {
    fewer_registers();
    // Rows [64 w, 64 w + 64) of each block, LPR lanes a row, 16 bytes a lane.
    constexpr int LPR = D / 8, PER = 32 / LPR;
    const int r0 = (warp - LOADER) * 64 + lane / LPR, ch = lane % LPR;
    int use = 0;
    bool ok = true;
    while (ok && next_run(A, P, sp, runs, walk, R)) {
      const AttendUnit& U = R.U;
      for (int x = 0; ok && x < 2; ++x) {
        if (!R.has(x)) continue;
        const int place = use % SM::QS;
        if (!wait_all(&q_empty[place], (uint32_t)(use / SM::QS) & 1u ^ 1u, abort_)) { ok = false; break; }
        const uint32_t dst = smem_u32(sm + place * SM::TILE + (ch / 8) * SM::HALF);
#pragma unroll 4
        for (int i = 0; i < 64; i += PER) {
          const int r = r0 + i, brow = R.first_row(x) + r, row = U.row0 + brow;
          const bool in = brow < U.rows;
          const int tok = J.by_r(row), j = row - tok * J.r;
          const uint8_t* src =
              A.q + (in ? ((int64_t)(J.off[U.b] + tok) * J.stride + (int64_t)(U.h * J.r + j) * D) * 2 + ch * 16 : 0);
          const uint32_t to = dst + r * 128 + ((ch % 8) ^ (r % 8)) * 16;
          if (A.qvec) {
            copy_async16(to, src, in);
          } else {
            const uint4 w = in ? load_plain16(src, false) : make_uint4(0, 0, 0, 0);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w)
                         : "memory");
          }
        }
        copies_wait();
        fence_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_full[place]);
        ++use;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFTMAX_REGS));
    const int x = warp / 4, lrow = threadIdx.x % 128;   // block, its row
    const uint32_t lanes = (uint32_t)((warp % 4) * 32) << 16;
    const uint32_t scol = tmem + lanes + x * BK, ocol = tmem + lanes + SM::O_COL + x * SM::O_STRIDE;
    const uint64_t al2 = pk2(A.alpha, A.alpha);
    uint32_t sph = 0, fph = 1;                           // phases of s_ready, and of the o_free before
    bool ok = true;
    while (ok && next_run(A, P, sp, runs, walk, R)) {
      if (!R.has(x)) continue;
      const int end = block_end(A, R, x), s0 = R.s0;
      const int brow = R.first_row(x) + lrow;
      const int lim = brow < R.U.rows ? keys_of(A.causal, R.U.len, R.U.n, J.by_r(R.U.row0 + brow)) : 0;
      const int all = __reduce_min_sync(0xffffffffu, lim);   // keys that every row of the warp sees
      float m = -INFINITY, l = 0.f;
      for (int s = s0; s < end; ++s) {
        if (!wait_all(&s_ready[x], sph, abort_)) { ok = false; break; }
        sph ^= 1u;
        fence_after();
        // Half a row at a time; the second half is read again: 128 values and the rest do not fit
        // in the registers.
        float v[64];
        const bool cut = s * BK + BK > all;              // keys that some row of the warp does not see
        auto half = [&](int i) {
          ld32(scol + i, v);
          ld32(scol + i + 32, v + 32);
          tmem_wait_ld();
          pin32(v);
          pin32(v + 32);
          if (cut) {
#pragma unroll
            for (int j = 0; j < 64; j += 32) {
              const int n = lim - (s * BK + i + j);
              const uint32_t seen = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
#pragma unroll
              for (int k = 0; k < 32; ++k)
                if (!(seen >> k & 1u)) v[j + k] = -INFINITY;
            }
          }
        };
        half(64);
        float top = max_of<64>(v);
        half(0);
        top = fmaxf(top, max_of<64>(v)) * A.alpha;
        // raises the maximum where some row's passes it by enough
        if (__any_sync(0xffffffffu, top > m + kRaise)) {
          const float mn = fmaxf(m, top), f = m == -INFINITY ? 0.f : fast_exp2(m - mn);
          m = mn;
          l *= f;
          if (s != s0) {
#pragma unroll 1
            for (int i = 0; i < D; i += 16) {
              float o[16];
              tmem_ld16(ocol + i, o);
              tmem_wait_ld16(o);
              uint32_t w[16];
#pragma unroll
              for (int k = 0; k < 16; ++k) w[k] = __float_as_uint(o[k] * f);
              st16(ocol + i, w);
            }
          }
        }
        const float mu = m == -INFINITY ? 0.f : m;
        const uint64_t mu2 = pk2(-mu, -mu);
        uint64_t sum2[2] = {pk2(0.f, 0.f), pk2(0.f, 0.f)};
#pragma unroll
        for (int i = 0; i < BK; i += 32) {
          if (i == 64) half(64);
          uint32_t w[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float a, b;
            upk2(ffma2(pk2(v[i % 64 + 2 * k], v[i % 64 + 2 * k + 1]), al2, mu2), a, b);
            a = fast_exp2(a);
            b = fast_exp2(b);
            sum2[k % 2] = fadd2(sum2[k % 2], pk2(a, b));
            w[k] = pack_bf16(a, b);
          }
          st16(scol + i / 2, w);
        }
        float a, b;
        upk2(fadd2(sum2[0], sum2[1]), a, b);
        l += a + b;
        wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_ready[x]);
      }
      if (!ok) break;
      // the finishers have read what the block's last run left here
      if (!wait_all(&o_free[x], fph, abort_)) break;
      fph ^= 1u;
      hd.ml[x][lrow] = make_float2(m, l);
      __syncwarp();
      if (lane == 0) mbar_arrive(&l_ready[x]);
    }
  }

  fence_before();
  __syncthreads();
  if (warp == ISSUER) tmem_dealloc(tmem, 512);
  if (threadIdx.x == 0 && hd.abort_flag) set_status(J.status, kStatusTimeout);
}

template <int D>
cudaError_t launch(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  using SM = PromptSmem<D>;
  const CacheJob& J = A.c;
  CUtensorMap kmap, vmap;
  const uint64_t rows = J.off[J.B], cols = (uint64_t)J.Hkv * D, pitch = A.kv_stride * 2;
  if (!make_tmap_bf16_3d(&kmap, J.kp, cols, rows, 1, pitch, rows * pitch, BK) ||
      !make_tmap_bf16_3d(&vmap, J.vp, cols, rows, 1, pitch, rows * pitch, BK))
    return cudaErrorInvalidValue;
  const cudaError_t e =
      cudaFuncSetAttribute(attend_prompt_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::BYTES);
  if (e != cudaSuccess) return e;
  return launch_kernel(attend_prompt_kernel<D>, dim3(P.workers), SM::NT, SM::BYTES, st, true, 0, kmap, vmap, A, P);
}

}  // namespace

cudaError_t launch_prompt_umma(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  return A.c.d == 128 ? launch<128>(A, P, st) : launch<64>(A, P, st);
}

}  // namespace mmshift
