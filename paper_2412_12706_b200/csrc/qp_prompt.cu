// Attention weight the keys of a prompt have received from its queries (qp_prompt_weights).
//
//   W[j] = sum over the G query heads h and the rows i with q_start + i >= j of 2^(t[h,i,j] - lse[h,i]),
//   t = q[h,i].k[j] log2(e) / sqrt(D),   lse[h,i] = log2 sum_{j <= q_start+i} 2^t[h,i,j].
//
// A row's normaliser needs all of the row before any column can be summed and the L^2 logits are never stored, so the product
// Q K^T is formed twice (sweep 1: lse, sweep 2: column sums), each time on the 5th-generation tensor cores.  The bound of a
// sweep is per 128 x 128 tile of logits: 16384 exponentials, 1024 clocks of the SM's 16-per-clock unit, against 512 clocks of
// the tensor cores (D = 128) and 32 KB of operand.  From that follow
//   - one block per SM with FOUR operand tiles resident in shared memory (sweep 1: query tiles; sweep 2: key tiles) and the
//     other operand streamed past them by TMA, so a streamed tile of 32 KB feeds four tiles of logits: one tile per block of
//     logits would ask the L2 cache for 15 TB/s;
//   - four reading groups of four warps, one per resident tile and 128-column tensor-memory buffer.  A thread owns one row of
//     its resident tile (a query in sweep 1, a key in sweep 2: the operands are swapped), so running sums are thread-local:
//     no shuffles, no atomics, a fixed order.  While one group waits for its next product the other three compute;
//   - part of the exponentials evaluated on the FMA pipe (ex2_poly2), two at a time with packed 32-bit arithmetic;
//   - sweep 1 without a running maximum: a row's reference is renewed only when a chunk's sum leaves the range in which
//     nothing can overflow, which the sum itself shows.
// Tiles above the diagonal are skipped, for each group on its own.  The work of all quads of resident tiles, end to end, is cut
// into one run per SM (see Plan); a quad that several runs share leaves partial results, which two small kernels add in a fixed
// order.
//
// Measured in a replayed graph: 8192 tokens of 32 heads over 8 (D = 128) 0.56 ms = 0.98 PFLOP/s of products (0.54 in short runs, before
// the limit is reached), the exponential unit
// 73 to 76 % busy, the tensor pipe 48 to 50 %, at the GPU's power limit; 1999 queries behind 14301 keys, 64 heads over 8, 1.07 ms;
// 1024 tokens of 8 heads over 2 (D = 64) 19 us, four launches one after another.
#include <algorithm>

#include "qp_mma.cuh"
#include "qp_tc.cuh"

namespace qp {

namespace {

constexpr int PW_GROUPS = 4, PW_STAGES = 3;
constexpr int PW_READ_WARPS = 4 * PW_GROUPS;
constexpr int PW_THREADS = (PW_READ_WARPS + 2) * 32;   // + the copy warp and the MMA warp
constexpr uint32_t PW_TMEM_COLS = 512;

// One sweep's work.  Resident tiles come in quads: sweep 1, tile r of a KV head = query tile r / G of its query head r % G;
// sweep 2, tile r = keys 128 r ..  A quad's streamed tiles are numbered 0 .. quad_steps - 1 (sweep 1: key tiles from the
// start; sweep 2: for each query head, the query tiles from the first that sees the quad).  The quads of all (batch, KV head)
// lie on one line, each as PW_SWITCH places that stand for fetching its resident tiles and then its steps; block i of `runs` does
// the steps in one of `runs` equal shares of it, so every block is done at the same time whatever the shape.
// (Pieces of one length, one to a block, dealt out by the hardware: 593 us for 8192 tokens of 32 heads over 8, 1080 us for the
// last 1999 of 16k of 64 over 8; the line: 562 and 1070, at 1.73 GHz and the GPU's power limit.  1, 2 or 3 places for a fetch
// differ by less than 2 %.)
constexpr int PW_SWITCH = 1;
struct Plan {
  int Hq, Hkv, G, L, nq, q_start, n;   // n = q_start + nq
  int nqt, nquads, runs, max_parts;    // max_parts: runs that can share a quad
  long long head_len, length;          // places of a (batch, KV head), of all
  long long run_len;                   // of a run; the first `longer` runs have one more
  int longer;
};

__host__ __device__ inline int quad_steps(int pass, const Plan& p, int quad) {
  if (pass == 1) {
    const int t = min(p.nqt - 1, (4 * quad + 3) / p.G);
    return (p.q_start + min(p.nq, (t + 1) * 128) - 1) / 128 + 1;
  }
  return p.G * (p.nqt - max(0, 512 * quad - p.q_start) / 128);
}
__device__ __forceinline__ long long run_start(const Plan& p, int i) { return p.run_len * i + min(i, p.longer); }
// places divided by a length: 32 bits for all but the very longest
__device__ __forceinline__ int place_div(const Plan& p, long long x, long long len) {
  return p.length <= 0x7fffffff ? (int)((unsigned)x / (unsigned)len) : (int)(x / len);
}
__device__ __forceinline__ int run_of(const Plan& p, long long place) {
  const long long split = (p.run_len + 1) * p.longer;
  return place < split ? place_div(p, place, p.run_len + 1) : p.longer + place_div(p, place - split, p.run_len);
}
// the quad that holds place `at` of a head, or with at < 0 quad `want`; its first place.  Called by whole warps.
__device__ __forceinline__ int find_quad(int pass, const Plan& p, long long at, int want, long long& first) {
  const int lane = threadIdx.x & 31;
  long long base = 0;
  for (int q0 = 0;; q0 += 32) {
    const int q = q0 + lane, len = q < p.nquads ? quad_steps(pass, p, q) + PW_SWITCH : 0;
    int inc = len;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    const unsigned past = __ballot_sync(0xffffffffu, at < 0 ? q >= want : base + inc > at);
    if (past || q0 + 32 >= p.nquads) {
      const int src = past ? __ffs(past) - 1 : 31;
      first = base + __shfl_sync(0xffffffffu, inc - len, src);
      return q0 + src;
    }
    base += __shfl_sync(0xffffffffu, inc, 31);
  }
}

enum : int { PB_A_FULL = 0, PB_A_EMPTY = PW_GROUPS, PB_S_FULL = 2 * PW_GROUPS, PB_S_EMPTY = PB_S_FULL + PW_STAGES, PB_T_FULL = PB_S_EMPTY + PW_STAGES,
             PB_T_EMPTY = PB_T_FULL + PW_GROUPS, PB_COUNT = PB_T_EMPTY + PW_GROUPS };

// pair `i` of a chunk: one of every PW_POLY through ex2_poly2, the others through the hardware unit (8192 tokens of 32 heads
// over 8, none / 1 of 8 / 1 of 4 / 3 of 8: 668 / 624 / 614 / 630 us)
constexpr int PW_POLY = 4;
template <bool TOP>
__device__ __forceinline__ uint64_t ex2_pair(uint64_t x, int i) {
  if (i % PW_POLY == 0) return ex2_poly2<TOP>(x);
  float a, b;
  unpack2(x, a, b);
  return pack2(ex2a(a), ex2a(b));
}

// sweep 1, 32 logits of a row that sees them all: s += sum 2^(t - m).  The reference m is one of the row's own logits, so the
// true sum is at least 1 and terms that vanish do not matter; a sum above 2^40 renews it (a term is clamped at or reaches at
// least 2^126 before anything can overflow unnoticed).
__device__ __forceinline__ bool fold_row_all(const uint32_t (&r)[32], float scale_log2, float m, float& s) {
  const uint64_t sc = pack2(scale_log2, scale_log2);
  const uint64_t nm = pack2(-m, -m);
  uint64_t acc0 = pack2(0.f, 0.f), acc1 = acc0;
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    acc0 = add2(acc0, ex2_pair<true>(fma2(pack2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), sc, nm), i));
    acc1 = add2(acc1, ex2_pair<true>(fma2(pack2(__uint_as_float(r[2 * i + 2]), __uint_as_float(r[2 * i + 3])), sc, nm), i + 1));
  }
  float a, b;
  unpack2(add2(acc0, acc1), a, b);
  const float sum = a + b;
  if (!(sum <= 1.0995116e12f)) return false;                    // 2^40; so for the first chunk (m = -inf), for inf and NaN
  s += sum;
  return true;
}
// the same with a renewed reference, for the columns up to lim only (col0: this chunk's first)
__device__ __forceinline__ void fold_row_any(const uint32_t (&r)[32], int col0, int lim, float scale_log2, float& m, float& s) {
  float cm = -INFINITY;
#pragma unroll
  for (int i = 0; i < 32; ++i) cm = fmaxf(cm, col0 + i <= lim ? __uint_as_float(r[i]) : -INFINITY);
  if (cm == -INFINITY) return;
  const float mn = fmaxf(m, cm * scale_log2);                   // scale > 0: max commutes with it
  float acc = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) acc += col0 + i <= lim ? ex2a(fmaf(__uint_as_float(r[i]), scale_log2, -mn)) : 0.f;
  s = fmaf(s, ex2a(m - mn), acc);
  m = mn;
}
// sweep 2: the sum of 32 rows' probabilities for this thread's key; lse: the rows' normalisers, negated (-inf: no such row)
__device__ __forceinline__ float fold_column(const uint32_t (&r)[32], const float* lse, float scale_log2) {
  const uint64_t sc = pack2(scale_log2, scale_log2);
  uint64_t acc0 = pack2(0.f, 0.f), acc1 = acc0;
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    const ulonglong2 l = *reinterpret_cast<const ulonglong2*>(lse + 2 * i);      // two pairs
    acc0 = add2(acc0, ex2_pair<false>(fma2(pack2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), sc, l.x), i));
    acc1 = add2(acc1, ex2_pair<false>(fma2(pack2(__uint_as_float(r[2 * i + 2]), __uint_as_float(r[2 * i + 3])), sc, l.y), i + 1));
  }
  float a, b;
  unpack2(add2(acc0, acc1), a, b);
  return a + b;
}
__device__ __forceinline__ float fold_column_masked(const uint32_t (&r)[32], const float* lse, int first, int rows, float scale_log2) {
  float acc = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) acc += i >= first && i < rows ? ex2a(fmaf(__uint_as_float(r[i]), scale_log2, lse[i])) : 0.f;
  return acc;
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}

// out: sweep 1, float2 (reference, sum) [bh][quad][part][512 rows]; sweep 2, float [part][bh][512 * quads] column sums
// neg_lse: -lse, [Bt * Hq][128 * nqt], -inf behind the last row
template <int PASS, int D>
__global__ void __launch_bounds__(PW_THREADS, 1)
prompt_sweep_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ Plan p, int BH,
                    float scale_log2, const float* __restrict__ neg_lse, void* __restrict__ out) {
  constexpr uint32_t OPER = 128 * D * 2;                // one operand tile: D/64 swizzled blocks of 16 KB
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t bars[PB_COUNT];
  __shared__ __align__(16) float s_lse[PW_STAGES][128];
  __shared__ uint32_t tmem_base_slot;
  __shared__ int give_up, s_quad;
  __shared__ long long s_first;

  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t sA = (smem_u32(smem_raw) + 1023u) & ~1023u, sS = sA + PW_GROUPS * OPER;
  const uint32_t bar0 = smem_u32(&bars[0]);
  auto bar = [&](int which, int i) { return bar0 + (uint32_t)(which + i) * 8u; };
  const volatile int* gu = &give_up;

  if (tid == 0) {
    for (int i = 0; i < PW_STAGES; ++i) {
      mbar_init(bar(PB_S_FULL, i), 1);
      mbar_init(bar(PB_S_EMPTY, i), PASS == 1 ? 1 : 1 + PW_READ_WARPS);   // the commit (and the readers of the stage's lse)
    }
    for (int i = 0; i < PW_GROUPS; ++i) {
      mbar_init(bar(PB_A_FULL, i), 1);
      mbar_init(bar(PB_A_EMPTY, i), 1);
      mbar_init(bar(PB_T_FULL, i), 1);
      mbar_init(bar(PB_T_EMPTY, i), 4);                                    // its warps
    }
    give_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (warp == PW_READ_WARPS + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_base_slot)),
                 "r"(PW_TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  const long long run0 = run_start(p, blockIdx.x), run1 = run_start(p, blockIdx.x + 1);
  const int bh0 = place_div(p, run0, p.head_len);
  if (warp == 0) {
    long long first;
    const int q = find_quad(PASS, p, run0 - bh0 * p.head_len, 0, first);
    if (lane == 0) { s_quad = q; s_first = bh0 * p.head_len + first; }
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem_base = tmem_base_slot;
  // This block's part of a quad, and the walk over them: every warp does it for itself.
  struct Part {
    int bh, quad, b, hk, step0, n_loc;
    int t0;                                               // sweep 2: first query tile of a head
    long long first;                                      // the quad's place
  };
  Part part{bh0, s_quad - 1, 0, 0, 0, 0, 0, s_first};     // (before the first)
  auto next_part = [&]() {                                // false: the run is done
    do {
      if (part.quad >= 0 && part.quad + 1 == p.nquads) {
        part.quad = -1;
        ++part.bh;
      }
      ++part.quad;
      const int steps = quad_steps(PASS, p, part.quad);
      if (part.first >= run1) return false;
      const long long s0 = part.first + PW_SWITCH;
      part.step0 = (int)(max(run0, s0) - s0);
      part.n_loc = (int)(min(run1, s0 + steps) - s0) - part.step0;
      part.first = s0 + steps;
    } while (part.n_loc <= 0);
    part.b = part.bh / p.Hkv;
    part.hk = part.bh % p.Hkv;
    part.t0 = PASS == 2 ? max(0, 512 * part.quad - p.q_start) / 128 : 0;
    return true;
  };
  // the resident tile of group g: does it exist
  auto group_valid = [&](int g) { return PASS == 1 ? (4 * part.quad + g) / p.G < p.nqt : 128 * (4 * part.quad + g) < p.n; };
  // sweep 1: the last streamed tile it needs; sweep 2: the first query tile of a head it needs (both never, if it does not exist)
  auto group_bound = [&](int g) {
    if (PASS == 1) return group_valid(g) ? (p.q_start + min(p.nq, ((4 * part.quad + g) / p.G + 1) * 128) - 1) / 128 : -1;
    return group_valid(g) ? max(0, 128 * (4 * part.quad + g) - p.q_start) / 128 : 0x7fffffff;
  };
  bool more = next_part();
  chain_enter();                                        // the launch's set-up overlaps the previous kernel's end

  int done = 0;                                         // streamed tiles of the parts before this one
  if (warp == PW_READ_WARPS) {
    // ---- copy warp
    int issued = 0, resident = 0;                       // resident: fetches of resident tiles so far, PW_GROUPS a part
    bool ok = true;
    for (int n = 0; ok && more; ++n, more = next_part()) {
      for (int j = 0; j < part.n_loc; ++j) {
        const int at = done + j, st = at % PW_STAGES;
        if (at >= PW_STAGES) ok = mbar_wait_warp(bar(PB_S_EMPTY, st), (uint32_t)((at / PW_STAGES - 1) & 1), gu);
        if (!ok) break;
        if (lane == 0) {
          mbar_expect_tx(bar(PB_S_FULL, st), OPER + (PASS == 2 ? 512 : 0));
          int y;
          if (PASS == 1) {
            y = part.bh * p.L + (part.step0 + j) * 128;
          } else {
            const int per = p.nqt - part.t0, s = part.step0 + j, bq = part.b * p.Hq + part.hk * p.G + s / per, t = part.t0 + s % per;
            y = bq * p.nq + t * 128;
            bulk_load(smem_u32(&s_lse[st][0]), neg_lse + ((size_t)bq * p.nqt + t) * 128, 512, bar(PB_S_FULL, st));
          }
#pragma unroll
          for (int kb = 0; kb < D / 64; ++kb)
            tma_load_2d(sS + st * OPER + kb * 16384, PASS == 1 ? &map_k : &map_q, kb * 64, y, bar(PB_S_FULL, st));
        }
        issued = at + 1;
        __syncwarp();
        for (int g = 0; j == 0 && g < PW_GROUPS; ++g) { // behind the first streamed tile: the resident ones
          if (n > 0) ok = mbar_wait_warp(bar(PB_A_EMPTY, g), (uint32_t)((n - 1) & 1), gu);
          if (!ok) break;
          if (lane == 0) {
            if (group_valid(g)) {
              const int r = 4 * part.quad + g;
              const int y = PASS == 1 ? (part.b * p.Hq + part.hk * p.G + r % p.G) * p.nq + r / p.G * 128 : part.bh * p.L + 128 * r;
              mbar_expect_tx(bar(PB_A_FULL, g), OPER);
#pragma unroll
              for (int kb = 0; kb < D / 64; ++kb)
                tma_load_2d(sA + g * OPER + kb * 16384, PASS == 1 ? &map_q : &map_k, kb * 64, y, bar(PB_A_FULL, g));
            } else {
              mbar_arrive(bar(PB_A_FULL, g));           // (one phase a part for every group)
            }
          }
          ++resident;
          __syncwarp();
        }
        if (!ok) break;
      }
      done += part.n_loc;
    }
    if (!ok) {
      give_up = 1;
      // the copies still on their way land in this block's shared memory: wait for them before it is given up
      auto landed = [&](uint32_t full, uint32_t parity) {
        for (uint32_t i = 0; i < TC_SPIN_LIMIT; ++i)
          if (mbar_try_wait(full, parity)) return;
      };
      for (int i = max(0, resident - PW_GROUPS); i < resident; ++i)
        landed(bar(PB_A_FULL, i % PW_GROUPS), (uint32_t)((i / PW_GROUPS) & 1));
      for (int j = max(0, issued - PW_STAGES); j < issued; ++j)
        landed(bar(PB_S_FULL, j % PW_STAGES), (uint32_t)((j / PW_STAGES) & 1));
    }
  } else if (warp == PW_READ_WARPS + 1) {
    // ---- MMA warp: streamed tile j against the resident tiles that need it
    constexpr uint32_t IDESC = instr_desc(128, 128);
    int uses[PW_GROUPS] = {}, bound[PW_GROUPS];
    bool ok = true;
    for (int n = 0; ok && more; ++n, more = next_part()) {
#pragma unroll
      for (int g = 0; g < PW_GROUPS; ++g) bound[g] = group_bound(g);
      int t = PASS == 2 ? part.t0 + part.step0 % (p.nqt - part.t0) : 0;   // sweep 2: query tile of the step
      for (int j = 0; j < part.n_loc && ok; ++j) {
        const int st = (done + j) % PW_STAGES;
        ok = mbar_wait_warp(bar(PB_S_FULL, st), (uint32_t)(((done + j) / PW_STAGES) & 1), gu);
#pragma unroll
        for (int g = 0; g < PW_GROUPS; ++g) {
          // (needed or not: a tile whose fetch may be under way is not handed back)
          if (ok && j == 0) ok = mbar_wait_warp(bar(PB_A_FULL, g), (uint32_t)(n & 1), gu);
          if (ok && (PASS == 1 ? part.step0 + j <= bound[g] : t >= bound[g])) {
            if (uses[g] > 0) ok = mbar_wait_warp(bar(PB_T_EMPTY, g), (uint32_t)((uses[g] - 1) & 1), gu);
            if (ok) {
              ++uses[g];
              asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
              const uint32_t a = uniform(desc_lo(sA + g * OPER, 1)), s = uniform(desc_lo(sS + st * OPER, 1));
              const uint32_t tm = uniform(tmem_base + g * 128), full = uniform(bar(PB_T_FULL, g));
              if (elect_one()) {
                umma_ss<false>(tm, a, s, IDESC);
#pragma unroll
                for (int k = 1; k < D / 16; ++k)
                  umma_ss<true>(tm, a + (k / 4) * 1024 + (k % 4) * 2, s + (k / 4) * 1024 + (k % 4) * 2, IDESC);
                umma_commit(full);
              }
              __syncwarp();
            }
          }
          const uint32_t idle = uniform(bar(PB_A_EMPTY, g));
          if (ok && j + 1 == part.n_loc && elect_one()) umma_commit(idle);
          __syncwarp();
        }
        const uint32_t empty = uniform(bar(PB_S_EMPTY, st));
        if (ok && elect_one()) umma_commit(empty);
        __syncwarp();
        if (PASS == 2 && ++t == p.nqt) t = part.t0;
      }
      done += part.n_loc;
    }
    // the last hand-back, which nobody waits for, has arrived before the block ends
    if (ok && done > 0) ok = mbar_wait_warp(bar(PB_S_EMPTY, (done - 1) % PW_STAGES), (uint32_t)(((done - 1) / PW_STAGES) & 1), gu);
    if (!ok) give_up = 1;
  } else {
    // ---- reading groups
    const int g = warp >> 2, rloc = (warp & 3) * 32 + lane;
    const uint32_t taddr = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + g * 128;
    int uses = 0;
    bool ok = true;
    for (; more; more = next_part()) {
      const int bound = group_bound(g), tq = PASS == 1 ? (4 * part.quad + g) / p.G : 0;
      float m_run = -INFINITY, s_run = 0.f;             // sweep 1: this thread's row; sweep 2: s_run = its key's sum
      int t = PASS == 2 ? part.t0 + part.step0 % (p.nqt - part.t0) : 0;
      for (int j = 0; j < part.n_loc && ok; ++j) {
        const int st = (done + j) % PW_STAGES, step = part.step0 + j;
        // sweep 2 hands the stage back below whether it needed it or not, and only once it has been filled: a group that
        // skips tiles must not run ahead of the ring
        if (PASS == 2) ok = mbar_wait_warp(bar(PB_S_FULL, st), (uint32_t)(((done + j) / PW_STAGES) & 1), gu);
        if (!ok) break;
        if (PASS == 1 ? step <= bound : t >= bound) {
          ok = mbar_wait_warp(bar(PB_T_FULL, g), (uint32_t)(uses & 1), gu);
          if (!ok) break;
          ++uses;
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
          bool all;                                     // every row of the tile sees every key of it
          int lim, rows = 128;                          // sweep 1: last column this row sees; sweep 2: first row that sees this key
          if (PASS == 1) {
            all = 128 * step + 127 <= p.q_start + 128 * tq;
            lim = min(p.q_start + 128 * tq + rloc, p.n - 1) - 128 * step;
          } else {
            const int key0 = 128 * (4 * part.quad + g);
            rows = p.nq - 128 * t;                      // (what lies behind a head's last row is the next head's, and may hold anything)
            all = key0 + 127 <= p.q_start + 128 * t && rows >= 128;
            // a query that is not finite has no normaliser: its tile takes the other path, because the polynomial clamps NaN away
            const float4 l = *reinterpret_cast<const float4*>(&s_lse[st][4 * lane]);
            all = all && __all_sync(0xffffffffu, fabsf(l.x + l.y + l.z + l.w) < INFINITY);
            lim = key0 + rloc - p.q_start - 128 * t;
          }
          auto fold = [&](const uint32_t (&r)[32], int c0) {
            if constexpr (PASS == 1) {
              if (!all || !fold_row_all(r, scale_log2, m_run, s_run)) fold_row_any(r, c0, lim, scale_log2, m_run, s_run);
            } else {
              const float* l = &s_lse[st][c0];
              s_run += all ? fold_column(r, l, scale_log2) : fold_column_masked(r, l, lim - c0, rows - c0, scale_log2);
            }
            __syncwarp();                               // the tensor-memory instructions want the whole warp
          };
          // a loop, not unrolled: the folds are long, and their code has to stay in the instruction cache
#pragma unroll 1
          for (int c0 = 0; c0 < 128; c0 += 32) {
            uint32_t v[32];
            tmem_ld32_issue(taddr + c0, v);
            tmem_wait(v);
            if (c0 == 96) {                               // the buffer is handed back before the last arithmetic
              asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
              __syncwarp();
              if (lane == 0) mbar_arrive(bar(PB_T_EMPTY, g));
            }
            fold(v, c0);
          }
        }
        if (PASS == 2) {
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(PB_S_EMPTY, st));
          if (++t == p.nqt) t = part.t0;
        }
      }
      done += part.n_loc;
      if (!ok) { give_up = 1; s_run = NAN; }            // a wait that ran out shows in what it was for
      if (group_valid(g)) {
        // the quad's first place is behind us by its steps: which of the runs that share it this one is
        const int nth = blockIdx.x - run_of(p, part.first - quad_steps(PASS, p, part.quad));
        if (PASS == 1)
          static_cast<float2*>(out)[(((size_t)part.bh * p.nquads + part.quad) * p.max_parts + nth) * 512 + tid] = make_float2(m_run, s_run);
        else
          static_cast<float*>(out)[((size_t)nth * BH + part.bh) * (512 * (size_t)p.nquads) + 512 * (size_t)part.quad + tid] = s_run;
      }
    }
  }

  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();                                      // every part is done with shared and tensor memory
  if (warp == PW_READ_WARPS + 1) {
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem_base), "r"(PW_TMEM_COLS) : "memory");
  }
}

// runs that share a quad.  Called by whole warps.
__device__ __forceinline__ int quad_parts(int pass, const Plan& p, int bh, int quad) {
  long long first;
  find_quad(pass, p, -1, quad, first);
  first += bh * p.head_len + PW_SWITCH;
  return run_of(p, first + quad_steps(pass, p, quad) - 1) - run_of(p, first) + 1;
}

// -lse of every row from the parts' (reference, sum) pairs, -inf for the padding rows of a head's last tile
// A launch of its own: a warp of sweep 2 that forms them for every streamed tile saves it, but is a chain of two reads and a loop
// per step (1024 tokens of 8 heads over 2: 19.4 -> 22.0 us, 8192 of 32 over 8: 565 -> 645 us).
__global__ void __launch_bounds__(256)
prompt_lse_kernel(const Plan p, const float2* __restrict__ stats, float* __restrict__ neg_lse) {
  const int i = blockIdx.x * 256 + threadIdx.x, bq = blockIdx.y, b = bq / p.Hq, hq = bq % p.Hq, h = hq % p.G;
  if (i >= p.nqt * 128) return;                         // (whole warps)
  const int bh = b * p.Hkv + hq / p.G, r = (i / 128) * p.G + h, quad = r / 4;
  const int parts = quad_parts(1, p, bh, quad);
  chain_enter();
  const float2* s = stats + (((size_t)bh * p.nquads + quad) * p.max_parts) * 512 + (r % 4) * 128 + (i & 127);
  float m = -INFINITY, z = 0.f;
  for (int c0 = 0; c0 < parts; c0 += 4) {
    float2 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = s[(size_t)min(c0 + k, parts - 1) * 512];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c0 + k < parts) {
        const float mn = fmaxf(m, v[k].x);
        z = v[k].x == -INFINITY ? z + v[k].y : z * exp2f(m - mn) + v[k].y * exp2f(v[k].x - mn);    // (a piece without visible keys: 0)
        m = mn;
      }
  }
  neg_lse[(size_t)bq * (p.nqt * 128) + i] = i < p.nq ? -(m + log2f(z)) : -INFINITY;
}

// weights from the parts' column sums, in the parts' order
__global__ void __launch_bounds__(256)
prompt_add_kernel(const Plan p, int BH, const float* __restrict__ part, int accumulate, float* __restrict__ weights) {
  const int j = blockIdx.x * 256 + threadIdx.x, bh = blockIdx.y;
  const int parts = j / 512 < p.nquads ? quad_parts(2, p, bh, j / 512) : 0;      // (the same for a whole block)
  chain_enter();
  if (j >= p.L) return;
  float* w = weights + (size_t)bh * p.L + j;
  if (j >= p.n) {
    if (!accumulate) *w = 0.f;
    return;
  }
  const size_t stride = (size_t)BH * (512 * (size_t)p.nquads);
  const float* s = part + (size_t)bh * (512 * (size_t)p.nquads) + j;
  float acc = 0.f;
  for (int c0 = 0; c0 < parts; c0 += 4) {
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = s[(size_t)min(c0 + k, parts - 1) * stride];
#pragma unroll
    for (int k = 0; k < 4; ++k) acc += c0 + k < parts ? v[k] : 0.f;
  }
  *w = accumulate ? *w + acc : acc;
}

// rows of D bf16 values as a matrix fetched in boxes of [128 rows x 64 columns] with the 128-byte swizzle; boxes past the end
// are filled with zeros
cudaError_t row_map(CUtensorMap* map, const void* base, long long rows, int D) {
  EncodeTiledFn enc = encode_tiled();
  if (!enc) return cudaErrorNotSupported;
  const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)D * 2};
  const cuuint32_t box[2] = {64, 128}, elem[2] = {1, 1};
  const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, elem,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

Plan make_plan(int pass, const PromptDims& d) {
  Plan p{};
  p.Hq = d.Hq; p.Hkv = d.Hkv; p.G = d.Hq / d.Hkv; p.L = d.L; p.nq = d.nq; p.q_start = d.q_start; p.n = d.q_start + d.nq;
  p.nqt = (d.nq + 127) / 128;
  p.nquads = pass == 1 ? (p.nqt * p.G + 3) / 4 : (p.n + 511) / 512;
  int longest = 0;
  for (int q = 0; q < p.nquads; ++q) {
    const int n = quad_steps(pass, p, q);
    longest = std::max(longest, n);
    p.head_len += n + PW_SWITCH;
  }
  p.length = p.head_len * (d.Bt * d.Hkv);
  p.runs = (int)std::min<long long>(p.length, sm_count());
  p.run_len = p.length / p.runs;
  p.longer = (int)(p.length % p.runs);
  p.max_parts = (int)std::min<long long>(longest, longest / p.run_len + 2);
  return p;
}

struct PromptWorkspace {
  size_t stats, lse, part, total;
};
PromptWorkspace carve(const PromptDims& d, const Plan& p1, const Plan& p2) {
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const size_t BH = (size_t)d.Bt * d.Hkv;
  PromptWorkspace w{};
  w.stats = 0;
  w.lse = w.stats + up(BH * p1.nquads * p1.max_parts * 512 * sizeof(float2));
  w.part = w.lse + up((size_t)d.Bt * d.Hq * p1.nqt * 128 * sizeof(float));
  w.total = w.part + up(BH * p2.max_parts * p2.nquads * 512 * sizeof(float));
  return w;
}

template <int PASS, int D>
cudaError_t launch_sweep(const CUtensorMap& q, const CUtensorMap& k, const Plan& p, int BH, float scale_log2, const float* lse,
                         void* out, cudaStream_t st) {
  constexpr size_t smem = (PW_GROUPS + PW_STAGES) * (size_t)128 * D * 2 + 1024;
  static unsigned char done[64] = {};
  const cudaError_t e = allow_smem(prompt_sweep_kernel<PASS, D>, smem, done);
  if (e != cudaSuccess) return e;
  return launch_chained(prompt_sweep_kernel<PASS, D>, dim3(p.runs), dim3(PW_THREADS), smem, st, q, k, p, BH, scale_log2,
                        lse, out);
}

}  // namespace

size_t prompt_workspace(const PromptDims& d) { return carve(d, make_plan(1, d), make_plan(2, d)).total; }

cudaError_t launch_prompt_weights(const void* Q, const void* K, const PromptDims& d, int accumulate, float* weights, void* ws,
                                  size_t ws_bytes, cudaStream_t st) {
  const Plan p1 = make_plan(1, d), p2 = make_plan(2, d);
  const PromptWorkspace w = carve(d, p1, p2);
  if (ws_bytes < w.total) return cudaErrorMemoryAllocation;       // (before anything is launched: the caller's "too small")
  char* base = static_cast<char*>(ws);
  float2* stats = reinterpret_cast<float2*>(base + w.stats);
  float *lse = reinterpret_cast<float*>(base + w.lse), *part = reinterpret_cast<float*>(base + w.part);
  const int BH = d.Bt * d.Hkv;
  const float scale_log2 = (float)(1.4426950408889634 / sqrt((double)d.D));
  CUtensorMap mq, mk;
  cudaError_t e = row_map(&mq, Q, (long long)d.Bt * d.Hq * d.nq, d.D);
  if (e != cudaSuccess) return e;
  e = row_map(&mk, K, (long long)BH * d.L, d.D);
  if (e != cudaSuccess) return e;
  e = d.D == 128 ? launch_sweep<1, 128>(mq, mk, p1, BH, scale_log2, lse, stats, st)
                 : launch_sweep<1, 64>(mq, mk, p1, BH, scale_log2, lse, stats, st);
  if (e != cudaSuccess) return e;
  e = launch_chained(prompt_lse_kernel, dim3((p1.nqt * 128 + 255) / 256, d.Bt * d.Hq), dim3(256), 0, st, p1, (const float2*)stats, lse);
  if (e != cudaSuccess) return e;
  e = d.D == 128 ? launch_sweep<2, 128>(mq, mk, p2, BH, scale_log2, lse, part, st)
                 : launch_sweep<2, 64>(mq, mk, p2, BH, scale_log2, lse, part, st);
  if (e != cudaSuccess) return e;
  return launch_chained(prompt_add_kernel, dim3((d.L + 255) / 256, BH), dim3(256), 0, st, p2, BH, (const float*)part, accumulate, weights);
}

}  // namespace qp
