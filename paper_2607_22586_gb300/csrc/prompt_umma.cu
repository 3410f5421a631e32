// Attention over whole prompts of bfloat16 rows on the 5th-generation tensor cores
// (tcgen05 + TMA + TMEM).
//
// Tiles of 256 query rows (two blocks of 128, a token's heads next to one another) over tiles of
// 128 keys, S = Q K^T and O += P V as in the chunk kernel (attend_umma.cu): S and P in
// tensor memory, one softmax thread a row. Prompts have many tiles of few keys (a prompt of
// 1000 tokens and seven heads a KV head has 28 tiles, of 5 key tiles on average), so a
// run's start and end are other warps' work, and the products go on from run to run:
//   warps 0-7   softmax, a warpgroup a block;
//   warp 8      TMA producer of K and V tiles, which works the runs out for all;
//   warp 9      MMA issuer: a block's first S of the next run follows its last P V;
//   warp 10     Q of the next blocks into a ring of three places;
//   warp 11     cleans V where a tile is masked;
//   warps 12-15 take O out: 104 registers a thread.
// A block has as many whole tokens as fit in 128 rows (126 rows of seven heads each), so that one
// TMA box of their heads fills it; rows behind them are computed and dropped.
// The issuer's loop has conditions and bounds that the compiler knows to be the same in all lanes (votes and
// reductions, not loaded values): 32,768 tokens of 28 heads 4.9 to 5.3 ms (6.33). What all roles need of a run
// is in shared memory, and their code is kept short (16 ragged prompts 206 -> 160 us when it was shortened).
// K's and V's rows are tokens apart: a tile is one box of 128 rows. Rows behind a prompt's last
// are the next prompt's: a zero weight times a NaN there would be a NaN, so in tiles that hold
// keys which some row does not attend to, values that are not finite are set to zero
// for the product and added to the rows that do attend to them at the end.
// Every wait is bounded; a role that gives up ends the CTA as score_umma.cu says.
#include <algorithm>
#include <climits>

#include "attend_umma.cuh"

namespace mmshift {
namespace {

using namespace umma;

constexpr int PRODUCER = 8, ISSUER = 9, LOADER = 10, CLEANER = 11, FINISHER = 12;   // first warps of the roles
// Registers a thread of the softmax warpgroups and of the others: in all as many as at the launch.
constexpr int SOFTMAX_REGS = 152, OTHER_REGS = 104;

// Start: everything before in the stream is done, and the next kernel may take its place.
__device__ __forceinline__ void prompt_start() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// A run, as the roles need it: key tiles [s0, s1) of a unit. The producer works it out once for all.
struct PromptRun {
  int64_t slot;          // its first row's place for partial sums, -1 if the run has all of the unit's keys
  int tok0, h;           // the request's first token; KV head
  int n, row0, rows;     // the request's tokens; the tile's first row, its rows
  int s0, s1;
  int end[2];            // tiles [s0, end) are the block's: rows in front may see fewer keys
  int least;             // keys that every row sees
  int seq;               // pages: the group's sequence
  int blocks, use;       // bit b: block b has rows; its Q is use + (blocks == 3 ? b : 0)
};
__device__ __forceinline__ bool has(const PromptRun& r, int b) { return r.blocks >> b & 1; }
// The first row of block b in the tile; blocks have A.block_rows rows.
__device__ __forceinline__ int first_row(const AttendJob& A, const PromptRun& r, int b) {
  return r.blocks == 3 ? b * A.block_rows : 0;
}
__device__ __forceinline__ int q_use(const PromptRun& r, int b) { return r.use + (r.blocks == 3 ? b : 0); }
// Keys of the prompt's token tok.
__device__ __forceinline__ int keys_at(const AttendJob& A, const PromptRun& r, int tok) { return A.causal ? tok + 1 : r.n; }

template <int D>
struct PromptSmem {
  static constexpr int NT = 512;
  static_assert(256 * (SOFTMAX_REGS + OTHER_REGS) <= 512 * 128, "more registers than the launch has");
  static constexpr int HALVES = D / 64;
  static constexpr int HALF = BK * 128;              // 64 columns of 128 rows
  static constexpr int TILE = HALVES * HALF;         // a block of Q, a tile of K or V
  static constexpr int QS = 3;                       // blocks of Q
  static constexpr int RUNS = 4;                     // of the ring of runs
  static constexpr int READERS = 15;                 // warps that read it: all but the producer
  static constexpr int STAGES = D == 64 ? 8 : 4;
  // Before the tiles: barriers and what roles tell one another. All of the CTA's shared memory is
  // asked for, and none declared besides, so the tiles' alignment costs nothing.
  struct Head {
    uint64_t full[STAGES], empty[STAGES], q_full[QS], q_empty[QS];
    uint64_t s_ready[2], p_ready[2], o_ready[2], o_free[2], l_ready[2], v_ask, v_clean, drain;
    uint64_t run_full[RUNS], run_empty[RUNS];
    PromptRun run[RUNS];
    union {
      AttendScan<NT, 1> scan;          // before the roles begin
      float2 ml[2][BQ];                // a block's rows: maximum (base 2) and sum of weights
    };
    uint32_t tbase;
    int abort_flag, odd_flag;
  };
  static constexpr int BYTES = 227 * 1024;
  static_assert((QS + STAGES) * TILE + 3 * 1024 <= BYTES && sizeof(Head) <= 3 * 1024, "shared memory");
  static constexpr uint32_t O_COL = 256, O_STRIDE = D;
};

// The part of a row's sums that comes from values that are not finite, of columns
// [d0, d0 + 32): added with the row's weights, key by key. Rare, so slow.
template <int D>
__device__ __forceinline__ void add_not_finite(const AttendJob& A, const PromptRun& r, int tok, int j, float m, int d0,
                                               float* o) {
  const CacheJob& J = A.c;
  const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(A.q) + (size_t)(r.tok0 + tok) * J.stride +
                           (size_t)(r.h * J.r + j) * D;
#pragma unroll 1
  for (int t = max(r.s0, r.least / BK) * BK; t < min(r.s1 * BK, keys_at(A, r, tok)); ++t) {
    const size_t at = (size_t)(r.tok0 + t) * A.kv_stride + (size_t)r.h * D;
    const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(J.vp) + at + d0;
    bool any = false;
#pragma unroll 1
    for (int i = 0; i < 32; ++i) any |= !isfinite(to_f32(v[i]));
    if (!any) continue;
    const __nv_bfloat16* k = reinterpret_cast<const __nv_bfloat16*>(J.kp) + at;
    float s = 0.f;
#pragma unroll 1
    for (int i = 0; i < D; ++i) s = fmaf(to_f32(q[i]), to_f32(k[i]), s);
    const float p = fast_exp2(fmaf(s, A.alpha, -m));
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float x = to_f32(v[i]);
      if (!isfinite(x)) o[i] += p * x;
    }
  }
}

__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS)); }
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFTMAX_REGS)); }

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

// 32 bytes of a row at once where the address allows.
__device__ __forceinline__ void store32(uint8_t* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// PAGED: K and V are pages of a cache, which every row of a group of requests sees as a whole (the
// keys are whole pages, all in the pool): nothing is masked but what a box of no page fills with
// zeros, and results are sums.
template <int D, bool PAGED>
__global__ void __launch_bounds__(PromptSmem<D>::NT, 1) attend_prompt_kernel(const __grid_constant__ CUtensorMap qmap,
                                                              const __grid_constant__ CUtensorMap kmap,
                                                              const __grid_constant__ CUtensorMap vmap,
                                                              const __grid_constant__ AttendJob A,
                                                              const __grid_constant__ AttendPlan P,
                                                              const __grid_constant__ PromptOrder O) {
  using SM = PromptSmem<D>;
  extern __shared__ __align__(16) unsigned char smraw[];
  typename SM::Head& hd = *reinterpret_cast<typename SM::Head*>(smraw);
  unsigned char* sm = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smraw) + sizeof(typename SM::Head) + 1023) & ~uintptr_t(1023));
  unsigned char* ring = sm + SM::QS * SM::TILE;
  uint64_t *const full = hd.full, *const empty = hd.empty, *const q_full = hd.q_full, *const q_empty = hd.q_empty;
  uint64_t *const s_ready = hd.s_ready, *const p_ready = hd.p_ready, *const o_ready = hd.o_ready;
  uint64_t *const o_free = hd.o_free, *const l_ready = hd.l_ready;
  if (sm + (SM::QS + SM::STAGES) * SM::TILE > smraw + SM::BYTES) {   // the base is not where it always is
    if (threadIdx.x == 0) set_status(A.c.status, kStatusTimeout);
    return;
  }
  // Every role passes all fills of the barriers that it waits for, in order, and none runs ahead of
  // the wait of another by more than one: a parity says which fill is meant.
  volatile int* abort_ = &hd.abort_flag;
  const CacheJob& J = A.c;
  // known to be the same in all lanes, as the issuer's loop: 32,768 tokens of 28 heads 5.3 ms (6.0 without)
  const int warp = uniform(threadIdx.x / 32), lane = threadIdx.x % 32;

  if (threadIdx.x == 0) {
    hd.abort_flag = hd.odd_flag = 0;
    for (int s = 0; s < SM::STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < SM::QS; ++s) {
      mbar_init(&q_full[s], 1);
      mbar_init(&q_empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_ready[i], 1);
      mbar_init(&p_ready[i], 4);     // a warpgroup's warps
      mbar_init(&o_ready[i], 1);
      mbar_init(&o_free[i], 4);
      mbar_init(&l_ready[i], 4);
    }
    for (int s = 0; s < SM::RUNS; ++s) {
      mbar_init(&hd.run_full[s], 1);
      mbar_init(&hd.run_empty[s], SM::READERS);
    }
    mbar_init(&hd.v_ask, 1);
    mbar_init(&hd.v_clean, 1);
    mbar_init(&hd.drain, 1);
    fence_barrier_init();
    prefetch_tmap(&qmap);
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
  AttendSpan sp = {0, 0, 0, 0};
  if (!O.whole) sp = attend_span(A, P, &hd.scan);
  __syncthreads();                     // the scan's place is ml's from here on
  // A warp's walk over the runs. A run without blocks ends it.
  int at = 0;
  uint32_t at_phase = 0;
  auto next = [&](PromptRun& r) {
    if (!wait_all(&hd.run_full[at], at_phase, abort_)) return false;
    r = hd.run[at];
    __syncwarp();
    if (lane == 0) mbar_arrive(&hd.run_empty[at]);
    if (++at == SM::RUNS) { at = 0; at_phase ^= 1u; }
    return r.blocks != 0;
  };
  // Blocks of Q are used in the order of the runs, a run's first block first: use n lies in
  // place n % QS.
  // A warpgroup gives up or takes registers as a whole: all its warps execute the one instruction (PTX),
  // ahead of what their roles do.
  if (warp >= PRODUCER) {
    fewer_registers();
    if (warp == PRODUCER) {
      if (lane == 0) {
        int stage = 0, unit = sp.unit, out = 0, use = 0, singles = 0, round = 0;
        uint32_t phase = 0, out_phase = 0;
        int64_t before = sp.before;
        ArmedStages armed;
        bool ok = true;
        // The CTA's next run, into the ring; false where the ring's readers have given up.
        auto publish = [&](PromptRun& r) {
          r.blocks = 0;
          bool any = false;
          if (O.whole) {
            const int u = prompt_turn(O, gridDim.x, blockIdx.x, round++);
            any = u >= 0;
            if (any) {
              const PromptUnit x = prompt_unit(O, J.Hkv, A.causal, u);
              r.tok0 = J.off[x.b];
              r.h = x.h;
              r.n = J.off[x.b + 1] - r.tok0;
              r.row0 = x.tile * P.rows;
              r.rows = min(P.rows, r.n * J.r - r.row0);
              r.s0 = 0;
              r.s1 = (keys_at(A, r, J.by_r(r.row0 + r.rows - 1)) + BK - 1) / BK;
              r.slot = -1;
            }
          }
          int seq = 0;
          while (!any && before < sp.end) {
            const AttendUnit U = attend_unit(A, P, nullptr, unit);
            const int64_t first = before;
            attend_pieces(U, sp.begin, sp.end, first, r.s0, r.s1);
            before += U.cost;
            ++unit;
            any = r.s0 < r.s1;
            r.tok0 = J.off[U.b];
            r.h = U.h;
            r.n = PAGED ? U.keys : U.n;
            seq = U.b * J.Hkv + U.h;
            r.row0 = U.row0;
            r.rows = U.rows;
            r.slot = r.s0 == 0 && r.s1 == U.pieces ? -1 : (int64_t)attend_slot(blockIdx.x, sp.begin, first) * P.rows;
          }
          if (any) {
            r.least = PAGED ? INT_MAX / 2 : keys_at(A, r, J.by_r(r.row0));
            r.seq = seq;
            r.blocks = r.rows > A.block_rows ? 3 : 1 << (singles++ & 1);   // one block's rows: each in turn
            r.use = use;
            use += r.blocks == 3 ? 2 : 1;
            // at least a tile, so that the block has sums
            const int keys = keys_at(A, r, J.by_r(r.row0 + min(r.rows, A.block_rows) - 1));
            const int end = max(min(r.s1, (keys + BK - 1) / BK), r.s0 + 1);
            r.end[0] = r.blocks == 3 ? end : has(r, 0) ? r.s1 : r.s0;
            r.end[1] = has(r, 1) ? r.s1 : r.s0;
          }
          if (!wait_one(&hd.run_empty[out], out_phase ^ 1u, abort_)) return false;
          hd.run[out] = r;
          mbar_arrive(&hd.run_full[out]);
          if (++out == SM::RUNS) { out = 0; out_phase ^= 1u; }
          return true;
        };
        PromptRun r, n;
        ok = publish(r);
        while (ok && r.blocks) {
          ok = publish(n);                               // a run ahead, so that Q can be loaded
          const int row0 = r.tok0, col0 = r.h * D;
          const int32_t* const table = PAGED ? cache_table(J, r.seq) : nullptr;
          const int shift = PAGED ? min(J.page_shift, 7) : 7, boxes = BK >> shift;
          const int outside = J.n_pages << J.page_shift;   // a box from there on reads zeros
          // pages: a tile's boxes, asked for a tile ahead
          int32_t entry[PAGED ? 8 : 1];
          auto look_up = [&](int s) {
  #pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int t = s * BK + (i << shift);
              if (i < boxes) entry[PAGED ? i : 0] = s < r.s1 && t < r.n ? table[t >> J.page_shift] : -1;
            }
          };
          if (PAGED && ok) look_up(r.s0);
          for (int s = r.s0; ok && s < r.s1; ++s) {
  #pragma unroll 1
            for (int kv = 0; kv < 2; ++kv) {
              if (!wait_one(&empty[stage], phase ^ 1u, abort_)) { ok = false; break; }
              mbar_expect_tx(&full[stage], SM::TILE);
              const CUtensorMap* const map = kv ? &vmap : &kmap;
              unsigned char* const to = ring + stage * SM::TILE;
              if constexpr (PAGED) {
  #pragma unroll
                for (int i = 0; i < 8; ++i) {
                  if (i >= boxes) break;
                  const int got = page_row(entry[i], J.n_pages, J.page_shift, s * BK + (i << shift));
  #pragma unroll
                  for (int c = 0; c < SM::HALVES; ++c)
                    tma_load_3d(to + c * SM::HALF + (i << shift) * 128, map, &full[stage], c * 64, got < 0 ? outside : got, 0);
                }
              } else {
  #pragma unroll
                for (int c = 0; c < SM::HALVES; ++c)
                  tma_load_3d(to + c * SM::HALF, map, &full[stage], col0 + c * 64, row0 + s * BK, 0);
              }
              armed.arm(stage, phase);
              if (++stage == SM::STAGES) { stage = 0; phase ^= 1u; }
            }
            if (PAGED) look_up(s + 1);
          }
          r = n;
        }
        if (!armed.drain(full)) *abort_ = 1;
      }
      __syncwarp();
    } else if (warp == ISSUER) {
      const uint32_t id_s = idesc_bf16_f32(BQ, BK), id_o = idesc_bf16_f32(BQ, D) | (1u << 16);   // V: MN-major
      const uint64_t qd = sdesc_k_sw128(smem_u32(sm)), kd = sdesc_k_sw128(smem_u32(ring));
      const uint64_t vd = sdesc_mn_sw128(smem_u32(ring), SM::HALF);
      int stage = 0;
      uint32_t phase = 0, pp = 0, of = 0, vc = 0;        // of the ring, of block i's barriers (bit i), of v_clean
      bool ok = true, issued = false;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        ok = ok && wait_all(bar, parity & 1u, abort_);
        return ok;
      };
      auto step = [&] {
        if (++stage == SM::STAGES) { stage = 0; phase ^= 1u; }
      };
      auto commit = [&](uint64_t* bar) {
        if (elect_one()) mma_commit(bar);
        __syncwarp();
      };
      auto next_uniform = [&](PromptRun& r) {
        const bool any = __all_sync(0xffffffffu, next(r));
        r.s0 = uniform(r.s0);
        r.s1 = uniform(r.s1);
        r.end[0] = uniform(r.end[0]);
        r.end[1] = uniform(r.end[1]);
        r.least = uniform(r.least);
        r.blocks = uniform(r.blocks);
        r.use = uniform(r.use);
        return any;
      };
      // S of block x, whose Q is use q, with the K tile of the stage
      auto issue_s = [&](int x, int q, bool first, bool last) {
        const int place = q % SM::QS;
        if (first && !wait(&q_full[place], (uint32_t)(q / SM::QS))) return;
        fence_after();
        const uint64_t k = kd + (uint64_t)(stage * (SM::TILE >> 4)), at = qd + (uint64_t)(place * (SM::TILE >> 4));
        if (elect_one()) {
  #pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint64_t o = (uint64_t)(((ks / 4) * SM::HALF + (ks % 4) * 32) >> 4);
            mma_bf16(tmem + x * BK, at + o, k + o, id_s, ks > 0 ? 1u : 0u);
          }
          mma_commit(&s_ready[x]);
          if (last) mma_commit(&q_empty[place]);
        }
        __syncwarp();
        issued = true;
      };
      PromptRun r, n;
      bool have = next_uniform(r);
      if (have && wait(&full[stage], phase)) {
  #pragma unroll 1
        for (int x = 0; ok && x < 2; ++x)
          if (has(r, x)) issue_s(x, q_use(r, x), true, r.end[x] == r.s0 + 1);
        commit(&empty[stage]);
        step();
      }
      while (ok && have) {
        const bool more = next_uniform(n);
        const int masked = r.least / BK;                 // the first tile whose V is cleaned
        for (int s = r.s0; ok && s < r.s1; ++s) {
          // In order: P V of a tile reads P before S of the next tile (of this run or the next) takes
          // its place. While one block's products run, the other's softmax does.
          const int vst = stage;
          const bool last = s + 1 == r.s1;
          bool k_there = false, v_there = s < masked;
          if (!wait(&full[vst], phase)) break;
          if (!v_there && elect_one()) mbar_arrive(&hd.v_ask);
          __syncwarp();
          step();
  #pragma unroll 1
          for (int x = 0; x < 2; ++x) {
            const int end = x ? r.end[1] : r.end[0];
            if (s < end) {
              if (s == r.s0) {                           // the block's last O has been read
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
              const uint64_t v = vd + (uint64_t)(vst * (SM::TILE >> 4));
              if (elect_one()) {
  #pragma unroll
                for (int ks = 0; ks < BK / 16; ++ks)
                  mma_p(tmem + SM::O_COL + x * SM::O_STRIDE, tmem + x * BK + ks * 8, v + (uint64_t)((ks * 2048) >> 4), id_o,
                        s > r.s0 || ks > 0 ? 1u : 0u);
                if (s + 1 == end) mma_commit(&o_ready[x]);
                if (x || s >= r.end[1]) mma_commit(&empty[vst]);   // the run's last block has had the tile's V
              }
              __syncwarp();
            }
            if (last ? more && has(n, x) : s + 1 < end) {
              if (!k_there && !wait(&full[stage], phase)) break;
              k_there = true;
              const int next_end = x ? n.end[1] : n.end[0];
              issue_s(x, last ? q_use(n, x) : q_use(r, x), last, last ? next_end == n.s0 + 1 : s + 2 == end);
              if (!ok) break;
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
    } else if (warp >= FINISHER) {
      const int fw = warp - FINISHER;
      const uint32_t lanes = (uint32_t)(fw * 32) << 16;
      uint32_t oph = 0;                                    // bit x: phase of block x's o_ready
      bool ok = true;
      PromptRun r;
      while (ok && next(r)) {
  #pragma unroll 1
        for (int x = 0; ok && x < 2; ++x) {
          if (!has(r, x)) continue;
          const uint32_t ph = oph >> x & 1u;
          const int lrow = fw * 32 + lane, brow = first_row(A, r, x) + lrow, row = r.row0 + brow;
          const bool live = lrow < A.block_rows && brow < r.rows, whole = r.slot < 0, sums = PAGED || !whole;
          const int tok = J.by_r(row), j = row - tok * J.r;
          const int64_t orow = (int64_t)(r.tok0 + tok) * J.Hq + r.h * J.r + j, slot = whole ? orow : r.slot + brow;
          float* const po = PAGED && whole ? A.part : P.po;
          const uint32_t ocol = tmem + lanes + SM::O_COL + x * SM::O_STRIDE;
          if (!wait_all(&l_ready[x], ph, abort_) || !wait_all(&o_ready[x], ph, abort_)) { ok = false; break; }
          oph ^= 1u << x;
          fence_after();
          const float2 t = hd.ml[x][lrow];
          const float m = t.x, l = t.y;
          // set by this warp's lanes or those beside it, before they reported a tile clean whose product
          // is in O by now
          const bool fix = !PAGED && *reinterpret_cast<volatile int*>(&hd.odd_flag) != 0;
          const float f = l == 0.f ? 0.f : 1.f / l;
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
            if (!PAGED && fix) add_not_finite<D>(A, r, tok, j, m == -INFINITY ? 0.f : m, i, o);
            if (!sums) {
              uint8_t* const to = A.out + (orow * D + i) * 2;
  #pragma unroll
              for (int c = 0; c < 32; c += 16) {
                uint32_t w[8];
  #pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = l == 0.f ? 0u : pack_bf16(o[c + 2 * e] * f, o[c + 2 * e + 1] * f);
                if (A.ovec == 2) {
                  store32(to + 2 * c, w);
                } else {
                  store_row16(to + 2 * c, make_uint4(w[0], w[1], w[2], w[3]), A.ovec);
                  store_row16(to + 2 * c + 16, make_uint4(w[4], w[5], w[6], w[7]), A.ovec);
                }
              }
            } else {
  #pragma unroll
              for (int c = 0; c < 32; c += 8)
                store32(reinterpret_cast<uint8_t*>(po + slot * D + i + c), reinterpret_cast<const uint32_t*>(o + c));
            }
          }
          if (live) {
            if (sums) (PAGED && whole ? A.part_ml : P.pml)[slot] = t;
            else if (A.lse) A.lse[orow] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
          }
        }
      }
    } else if (warp == CLEANER) {
      uint32_t ask = 0;                                    // phase of v_ask
      int stage = 1;                                       // of the next tile's V
      bool ok = true;
      PromptRun r;
      while (ok && next(r)) {
        for (int s = r.s0; s < r.s1; ++s) {
          const int vs = stage, k0 = s * BK;
          stage = (stage + 2) % SM::STAGES;
          if (k0 + BK <= r.least) continue;
          if (!wait_all(&hd.v_ask, ask, abort_)) { ok = false; break; }
          ask ^= 1u;
          unsigned char* vt = ring + vs * SM::TILE;
          // Few tiles hold such values, so all of it is looked through before any is changed. A lane
          // has every 32nd of the tile's 16-byte chunks.
          constexpr int CH = SM::HALVES * 8, N = BK * CH / 32;    // chunks of a row, of a lane
          const int i0 = max(r.least - k0, 0) * CH;
          auto chunk = [&](int e) {
            const int i = e * 32 + lane, key = i / CH, ch = i % CH;
            return reinterpret_cast<uint4*>(vt + (ch / 8) * SM::HALF + key * 128 + (ch % 8) * 16);
          };
          uint32_t worst = 0;
  #pragma unroll 1
          for (int e0 = i0 / 32 / 8 * 8; e0 < N; e0 += 8) {
            uint4 w[8];
  #pragma unroll
            for (int e = 0; e < 8; ++e) {
              w[e] = make_uint4(0, 0, 0, 0);
              if ((e0 + e) * 32 + lane >= i0) w[e] = *chunk(e0 + e);
            }
  #pragma unroll
            for (int e = 0; e < 8; ++e) {
              constexpr uint32_t k = 0x7fff7fffu;
              worst = __vmaxu2(worst, __vmaxu2(__vmaxu2(w[e].x & k, w[e].y & k), __vmaxu2(w[e].z & k, w[e].w & k)));
            }
          }
          if (__any_sync(0xffffffffu, not_finite2(worst))) {
            const int keys = keys_at(A, r, J.by_r(r.row0 + r.rows - 1));
  #pragma unroll 1
            for (int e = 0; e < N; ++e) {
              const int i = e * 32 + lane;
              if (i < i0) continue;
              const uint4 w = *chunk(e);
              if (!(not_finite2(w.x) || not_finite2(w.y) || not_finite2(w.z) || not_finite2(w.w))) continue;
              if (k0 + i / CH < keys) *reinterpret_cast<volatile int*>(&hd.odd_flag) = 1;
              *chunk(e) = make_uint4(finite2(w.x), finite2(w.y), finite2(w.z), finite2(w.w));
            }
          }
          fence_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(&hd.v_clean);
        }
      }
    } else if (warp == LOADER) {
      bool ok = true;
      PromptRun r;
      ArmedStages armed;
      while (ok && next(r)) {
  #pragma unroll 1
        for (int x = 0; ok && x < 2; ++x) {
          if (!has(r, x)) continue;
          const int use = q_use(r, x), place = use % SM::QS, row0 = r.row0 + first_row(A, r, x);
          const uint32_t phase = (uint32_t)(use / SM::QS) & 1u;
          if (!wait_all(&q_empty[place], phase ^ 1u, abort_)) { ok = false; break; }
          unsigned char* const to = sm + place * SM::TILE;
          if (A.qbox) {                                    // the block begins with a token's first head
            if (lane == 0) {
              mbar_expect_tx(&q_full[place], A.block_rows * D * 2);
  #pragma unroll
              for (int c = 0; c < SM::HALVES; ++c)
                tma_load_3d(to + c * SM::HALF, &qmap, &q_full[place], c * 64, r.h * J.r, r.tok0 + J.by_r(row0));
            }
            armed.arm(place, phase);
          } else {                                         // rows that start anywhere, or a token's heads in several blocks
            constexpr int LPR = D / 8;                     // lanes of a row
  #pragma unroll 1
            for (int i = lane / LPR; i < BQ; i += 32 / LPR) {
              const int row = row0 + i, tok = J.by_r(row), ch = lane % LPR;
              const bool in = i < A.block_rows && row < r.row0 + r.rows;
              const uint8_t* src =
                  A.q + (in ? ((int64_t)(r.tok0 + tok) * J.stride + (int64_t)(r.h * J.r + row - tok * J.r) * D) * 2 + ch * 16 : 0);
              const uint4 w = in ? load_plain16(src, A.qvec) : make_uint4(0, 0, 0, 0);
              *reinterpret_cast<uint4*>(to + (ch / 8) * SM::HALF + i * 128 + ((ch % 8) ^ (i % 8)) * 16) = w;
            }
            fence_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(&q_full[place]);
          }
          __syncwarp();
        }
      }
      if (!armed.drain(q_full)) *abort_ = 1;
    }
  } else {
    more_registers();
    const int x = warp / 4, lrow = threadIdx.x % 128;   // block, its row
    const uint32_t lanes = (uint32_t)((warp % 4) * 32) << 16;
    const uint32_t scol = tmem + lanes + x * BK, ocol = tmem + lanes + SM::O_COL + x * SM::O_STRIDE;
    const uint64_t al2 = pk2(A.alpha, A.alpha);
    uint32_t sph = 0, fph = 1;                           // phases of s_ready, and of the o_free before
    bool ok = true;
    PromptRun r;
    while (ok && next(r)) {
      if (!has(r, x)) continue;
      const int s0 = r.s0, end = x ? r.end[1] : r.end[0], brow = first_row(A, r, x) + lrow;
      // rows that are none see everything, so that their warps need no mask, and raise no maximum: what
      // they hold is whatever lies behind the block's Q
      const bool live = lrow < A.block_rows && brow < r.rows;
      const int lim = live ? keys_at(A, r, J.by_r(r.row0 + brow)) : INT_MAX;
      const int all = __reduce_min_sync(0xffffffffu, lim);   // keys that every row of the warp sees
      float m = -INFINITY, l = 0.f;
      for (int s = s0; s < end; ++s) {
        if (!wait_all(&s_ready[x], sph, abort_)) { ok = false; break; }
        sph ^= 1u;
        fence_after();
        if (s * BK + BK > all) {                         // keys that some row of the warp does not see
#pragma unroll 1
          for (int i = max(all - s * BK, 0) / 32 * 32; i < BK; i += 32) {
            float y[32];
            uint32_t w[32];
            ld32(scol + i, y);
            tmem_wait_ld();
            pin32(y);
            const int n = lim - (s * BK + i);
            const uint32_t seen = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
#pragma unroll
            for (int k = 0; k < 32; ++k) w[k] = seen >> k & 1u ? __float_as_uint(y[k]) : 0xff800000u;
            st16(scol + i, w);
            st16(scol + i + 16, w + 16);
          }
          wait_st();
        }
        // Half a row at a time; the second half is read again: 128 values and the rest do not fit
        // in the registers.
        float v[64];
        auto half = [&](int i) {
          ld32(scol + i, v);
          ld32(scol + i + 32, v + 32);
          tmem_wait_ld();
          pin32(v);
          pin32(v + 32);
        };
        half(64);
        float top = max_of<64>(v);
        half(0);
        top = fmaxf(top, max_of<64>(v)) * A.alpha;
        // raises the maximum where some row's passes it by enough
        if (__any_sync(0xffffffffu, live && top > m + kRaise)) {
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
            // Weights go into the products as bfloat16, which is V's type and has to be theirs; their sum is of
            // float32 ones. Against 64 bits results are off by 0.0020 of their norm (16 ragged prompts) with
            // their own rounding to bfloat16, which alone is 0.0016.
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

template <int D, bool PAGED>
cudaError_t launch(AttendJob A, const AttendPlan& P, const PromptOrder& O, cudaStream_t st) {
  using SM = PromptSmem<D>;
  const CacheJob& J = A.c;
  CUtensorMap qmap, kmap, vmap;
  auto make = [&](CUtensorMap* m, const void* base) {
    if (PAGED) {
      const uint64_t rows = (uint64_t)J.n_pages << J.page_shift;
      return make_tmap_bf16_3d(m, base, D, rows, 1, D * 2, rows * D * 2, std::min(1 << J.page_shift, BK));
    }
    const uint64_t rows = J.off[J.B], cols = (uint64_t)J.Hkv * D, pitch = A.kv_stride * 2;
    return make_tmap_bf16_3d(m, base, cols, rows, 1, pitch, rows * pitch, BK);
  };
  if (!make(&kmap, J.kp) || !make(&vmap, J.vp)) return cudaErrorInvalidValue;
  qmap = kmap;                                           // not used where Q's rows are copied
  A.qbox = A.qvec && J.r <= BQ && J.stride < (int64_t)1 << 38;
  if (A.qbox &&
      !make_tmap_bf16_box(&qmap, A.q, D, J.Hq, J.off[J.B], D * 2, J.stride * 2, J.r, A.block_rows / J.r))
    return cudaErrorInvalidValue;
  const cudaError_t e =
      cudaFuncSetAttribute(attend_prompt_kernel<D, PAGED>, cudaFuncAttributeMaxDynamicSharedMemorySize, SM::BYTES);
  if (e != cudaSuccess) return e;
  return launch_kernel(attend_prompt_kernel<D, PAGED>, dim3(P.workers), SM::NT, SM::BYTES, st, true, 0, qmap, kmap, vmap, A, P,
                       O);
}

}  // namespace

cudaError_t launch_prompt_umma(const AttendJob& A, const AttendPlan& P, const PromptOrder& O, cudaStream_t st) {
  return A.c.d == 128 ? launch<128, false>(A, P, O, st) : launch<64, false>(A, P, O, st);
}

cudaError_t launch_common_umma(const AttendJob& A, const AttendPlan& P, cudaStream_t st) {
  const PromptOrder O = {};
  return A.c.d == 128 ? launch<128, true>(A, P, O, st) : launch<64, true>(A, P, O, st);
}

}  // namespace mmshift
