// Attention of a tree of drafted tokens over a packed cache, its tail and the drafts themselves (qp_decode_attn_tree).
//
// The T drafts' G query heads of one KV head are R = T G rows of one attention problem over N = n + n_tail + T tokens: with
// 4 R D flop per token against 2 D B / 8 bytes of cache the tensor cores are as much the bound as HBM, so both products run on
// tcgen05, the codes are expanded to fp16 once per (KV head, tile) whatever R is, and all T drafts cost one pass over the cache.
//
// A block owns up to 256 rows of one KV head and walks over a run of 128-token tiles; its parts talk through mbarriers only:
//   8 loader warps    tile j -> keys, then values, into a ring of 32 KB operand slots (128-byte swizzle).  Packed caches: words
//                     from global memory, one operand ahead in registers, to fp16 and into the slot.  16-bit caches: TMA, with
//                     the token count as the tensor's extent, so rows behind the last one arrive as zeros whatever the array
//                     holds there.  Tail and drafts form the last one or two tiles.
//   1 MMA warp        S[u] = Q[u] K_j^T into tensor memory; O[u] += P[u] V_j with P from tensor memory and V read with its rows
//                     as the contraction, so neither operand is transposed
//   2 softmax groups  u = 0, 1, four warps each, one row per thread: no shuffles.  S is read twice (maximum; exponentials); P
//                     overwrites the columns of S already read.  O is rescaled only when the maximum grows by more than 2^8
//                     (the weights then stay below 2^8 in 16 bits, relative precision unchanged).
// u is a tile of 128 rows when there are two, else (R <= 128) the parity of the token tile: two independent streams either
// way, so one group's exponentials run beside the other's products.
//
// The runs of one (KV head, row group) form a cluster: partial (max, sum, O) stay in shared memory, every CTA adds up its slice
// of the rows from all of them through distributed shared memory and writes it: one launch, no workspace but the error word.
// Order of additions fixed; every mbarrier wait bounded (see the score sweeps).
//
// Types: 16-bit caches multiply in bf16; packed ones in fp16 (2^-11 on a reconstructed value, against 2^-8 in bf16), tail,
// drafts and queries converted (exact but for |x| below 2^-14, off by at most 2^-25, or above 65504).  Logits, maxima, sums
// and O in 32 bits; the softmax weights enter the second product in 16 bits like its values.
#include <cooperative_groups.h>

#include <algorithm>
#include <cstring>

#include "qp_mma.cuh"
#include "qp_tc.cuh"

namespace qp {

namespace {

namespace cg = cooperative_groups;

constexpr int TR_SOFT = 8, TR_LOAD = 8;                          // warps
constexpr int TR_LOADERS = TR_LOAD * 32;
constexpr int TR_THREADS = (TR_SOFT + TR_LOAD + 1) * 32;
constexpr int TR_MAX_SLOTS = 6, TR_MAX_CLUSTER = 16;

enum : int { TB_FULL = 0, TB_EMPTY = TR_MAX_SLOTS, TB_S = 2 * TR_MAX_SLOTS, TB_P = TB_S + 2, TB_COUNT = TB_P + 2 };

struct TreeLaunch {
  TreeArgs a;
  int R, n_groups;           // rows per KV head, groups of up to 256 of them
  int two_rows;              // 1: stream u = row tile u of the group; 0: stream u = parity of the token tile
  int ctx_tiles, tiles;      // context tiles, and with the tail's and drafts'
  int slots, cluster;
};

// byte offset of 16-byte chunk c of row r in an operand tile of 128 rows
__device__ __forceinline__ uint32_t tile_off(int r, int c) {
  return (uint32_t)((c >> 3) * 16384 + (r >> 3) * 1024 + (r & 7) * 128 + (((c & 7) ^ (r & 7)) << 4));
}
__device__ __forceinline__ void sts128(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};\n" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint32_t half2_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;\n" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
// two bf16 values to two fp16 values
__device__ __forceinline__ uint32_t bf2_to_half2(uint32_t v) { return pack_half2(bf16lo(v), bf16hi(v)); }

// the codes at bit p of both 16-bit lanes of x, times s2, plus z2.  1024 + c 2^q is an fp16 value (c 2^q < 1024), the first
// multiply-add turns it into c exactly, the second rounds once.
template <int BITS>
__device__ __forceinline__ uint32_t code_pair(uint32_t x, int p, uint32_t s2, uint32_t z2) {
  constexpr uint32_t ones = (1u << BITS) - 1u;
  const int q = p & 7;
  const uint32_t h = ((p < 8 ? x : x >> 8) & ((ones | ones << 16) << q)) | 0x64006400u;
  const uint32_t down = (uint32_t)(15 - q) << 10;               // 2^-q
  const uint32_t off = 0x8000u | (uint32_t)(25 - q) << 10;      // -1024 * 2^-q
  return half2_fma(half2_fma(h, down | down << 16, off | off << 16), s2, z2);
}

// ---- loaders of one packed operand tile: fetch (global -> registers) and put (registers -> slot)
// Groups along the tokens (keys of the main path): an item is 8 channels x PT tokens, a word per channel.
template <int BITS, int D>
struct ColLoader {
  static constexpr int PER = 32 / BITS, PT = PER < 8 ? PER : 8, OCT = D / 8, ITEMS = (128 / PT) * OCT;
  static constexpr int PT_ITEMS = (ITEMS + TR_LOADERS - 1) / TR_LOADERS;
  uint32_t w[PT_ITEMS][8];
  uint4 s[PT_ITEMS], z[PT_ITEMS];
  __device__ __forceinline__ void fetch(const TreeArgs& a, int bh, int tok0, int lt) {
    const int g = a.group, wpg = g * BITS / 32;
#pragma unroll
    for (int k = 0; k < PT_ITEMS; ++k) {
      const int i = lt + k * TR_LOADERS, oct = i % OCT, tok = tok0 + i / OCT * PT;
      if (i >= ITEMS || tok >= a.n) continue;
      const size_t base = ((size_t)bh * (a.ns / g) + tok / g) * D + oct * 8;
      const uint32_t* src = static_cast<const uint32_t*>(a.kc) + base * wpg + (tok % g) / PER;
#pragma unroll
      for (int c = 0; c < 8; ++c) w[k][c] = __ldg(src + c * wpg);
      s[k] = __ldg(reinterpret_cast<const uint4*>(a.ks + base));
      z[k] = __ldg(reinterpret_cast<const uint4*>(a.kz + base));
    }
  }
  __device__ __forceinline__ void put(const TreeArgs& a, int tok0, int lt, uint32_t slot) {
#pragma unroll
    for (int k = 0; k < PT_ITEMS; ++k) {
      const int i = lt + k * TR_LOADERS, oct = i % OCT, row = i / OCT * PT;
      if (i >= ITEMS) continue;
      if (tok0 + row >= a.n) {                                  // (n is a multiple of 32: an item is inside or outside)
#pragma unroll
        for (int e = 0; e < PT; ++e) sts128(slot + tile_off(row + e, oct), make_uint4(0u, 0u, 0u, 0u));
        continue;
      }
      const uint32_t s2[4] = {s[k].x, s[k].y, s[k].z, s[k].w}, z2[4] = {z[k].x, z[k].y, z[k].z, z[k].w};
      const bool upper = BITS == 2 && ((tok0 + row) & 8);       // 16 tokens a word, 8 an item
#pragma unroll
      for (int half = 0; half < (PT * BITS > 16 ? 2 : 1); ++half) {
        uint32_t x[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = __byte_perm(w[k][2 * c], w[k][2 * c + 1], half || upper ? 0x7632 : 0x5410);
        constexpr int N = PT * BITS > 16 ? PT / 2 : PT;         // tokens in 16 bits
#pragma unroll
        for (int e = 0; e < N; ++e) {
          uint4 v;
          v.x = code_pair<BITS>(x[0], e * BITS, s2[0], z2[0]);
          v.y = code_pair<BITS>(x[1], e * BITS, s2[1], z2[1]);
          v.z = code_pair<BITS>(x[2], e * BITS, s2[2], z2[2]);
          v.w = code_pair<BITS>(x[3], e * BITS, s2[3], z2[3]);
          sts128(slot + tile_off(row + half * N + e, oct), v);
        }
      }
    }
  }
};
// Groups along the channels (values; keys quantized token by token): an item is 16 channels of one token.
template <int BITS, int D>
struct RowLoader {
  static constexpr int PIECES = D / 16, PT_ITEMS = 128 * PIECES / TR_LOADERS, W = BITS / 2;   // words of an item
  uint32_t w[PT_ITEMS][W];
  __half s[PT_ITEMS], z[PT_ITEMS];
  __device__ __forceinline__ void fetch(const TreeArgs& a, const void* codes, const __half* scale, const __half* zero, int bh, int tok0,
                                        int lt) {
#pragma unroll
    for (int k = 0; k < PT_ITEMS; ++k) {
      const int i = lt + k * TR_LOADERS, piece = i % PIECES, tok = tok0 + i / PIECES;
      if (tok >= a.n) continue;
      const size_t row = (size_t)bh * a.ns + tok, grp = row * (D / a.group) + piece * 16 / a.group;
      const uint32_t* src = static_cast<const uint32_t*>(codes) + (row * PIECES + piece) * W;
      if constexpr (W == 4) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(src));
        w[k][0] = v.x; w[k][1] = v.y; w[k][2] = v.z; w[k][3] = v.w;
      } else if constexpr (W == 2) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(src));
        w[k][0] = v.x; w[k][1] = v.y;
      } else {
        w[k][0] = __ldg(src);
      }
      s[k] = scale[grp];
      z[k] = zero[grp];
    }
  }
  __device__ __forceinline__ void put(const TreeArgs& a, int tok0, int lt, uint32_t slot) {
#pragma unroll
    for (int k = 0; k < PT_ITEMS; ++k) {
      const int i = lt + k * TR_LOADERS, piece = i % PIECES, row = i / PIECES;
      uint4 v[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
      if (tok0 + row < a.n) {
        const __half2 sh = __half2half2(s[k]), zh = __half2half2(z[k]);
        const uint32_t s2 = *reinterpret_cast<const uint32_t*>(&sh), z2 = *reinterpret_cast<const uint32_t*>(&zh);
        // a word's pair f holds channels f and f + 16/BITS; pairs f, f + 1 make the channel pairs (f, f+1) and the upper ones
        uint32_t c[8];                                          // channels (0,1) .. (14,15)
#pragma unroll
        for (int j = 0; j < W; ++j) {
          constexpr int U = 16 / BITS;
#pragma unroll
          for (int f = 0; f < U; f += 2) {
            const uint32_t p = code_pair<BITS>(w[k][j], f * BITS, s2, z2), q = code_pair<BITS>(w[k][j], (f + 1) * BITS, s2, z2);
            c[j * U + f / 2] = __byte_perm(p, q, 0x5410);
            c[j * U + U / 2 + f / 2] = __byte_perm(p, q, 0x7632);
          }
        }
        v[0] = make_uint4(c[0], c[1], c[2], c[3]);
        v[1] = make_uint4(c[4], c[5], c[6], c[7]);
      }
      sts128(slot + tile_off(row, 2 * piece), v[0]);
      sts128(slot + tile_off(row, 2 * piece + 1), v[1]);
    }
  }
};
// rows 128 x .. of the tail followed by the drafts, zeros behind them
template <int D, bool HALF>
__device__ __forceinline__ void put_extra(const TreeArgs& a, bool keys, int b, int hk, int bh, int x, int lt, uint32_t slot) {
  constexpr int PIECES = D / 16;
  const uint16_t* tail = static_cast<const uint16_t*>(keys ? a.k_tail : a.v_tail);
  const uint16_t* draft = static_cast<const uint16_t*>(keys ? a.k_draft : a.v_draft);
#pragma unroll
  for (int k = 0; k < 128 * PIECES / TR_LOADERS; ++k) {
    const int i = lt + k * TR_LOADERS, piece = i % PIECES, row = i / PIECES, e = 128 * x + row;
    uint4 v[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
    if (e < a.n_tail + a.T) {
      const uint16_t* src = e < a.n_tail ? tail + ((size_t)bh * a.group + e) * D
                                         : draft + (((size_t)b * a.T + (e - a.n_tail)) * a.Hkv + hk) * D;
      const uint4* p = reinterpret_cast<const uint4*>(src + piece * 16);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        v[j] = __ldg(p + j);
        if (HALF) v[j] = make_uint4(bf2_to_half2(v[j].x), bf2_to_half2(v[j].y), bf2_to_half2(v[j].z), bf2_to_half2(v[j].w));
      }
    }
    sts128(slot + tile_off(row, 2 * piece), v[0]);
    sts128(slot + tile_off(row, 2 * piece + 1), v[1]);
  }
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}

// the partial O of a stream in shared memory: 16-byte chunk c of row r, spread over the banks
template <int D>
__device__ __forceinline__ uint32_t part_off(int r, int c) { return (uint32_t)(r * (D * 4) + ((c ^ (r & (D / 4 - 1))) << 4)); }

template <int BITS, int D>
__global__ void __launch_bounds__(TR_THREADS, 1)
tree_kernel(const __grid_constant__ TreeLaunch p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
            int* __restrict__ error_word) {
  constexpr bool HALF = BITS < 16;
  constexpr uint32_t SLOT = 128 * D * 2;
  constexpr uint32_t FMT = HALF ? 0u : (1u << 7) | (1u << 10);  // both operands fp16 / bf16
  constexpr uint32_t ID_S = (1u << 4) | FMT | ((128u >> 3) << 17) | ((128u >> 4) << 24);
  constexpr uint32_t ID_O = (1u << 4) | FMT | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);   // B: rows contract
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t bars[TB_COUNT];
  __shared__ uint32_t tmem_base_slot;
  __shared__ int give_up;
  cg::cluster_group cluster = cg::this_cluster();

  const TreeArgs& a = p.a;
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int C = p.cluster, rank = blockIdx.x % C, item = blockIdx.x / C, rg = item % p.n_groups, bh = item / p.n_groups;
  const int b = bh / a.Hkv, hk = bh % a.Hkv, G = a.Hq / a.Hkv;
  const int row0 = rg * 256, rows = min(256, p.R - row0);       // of this group
  const int j0 = (int)((long long)p.tiles * rank / C), n_loc = (int)((long long)p.tiles * (rank + 1) / C) - j0;
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sQ = sbase, ring = sbase + (p.two_rows ? 2 : 1) * SLOT;
  const uint32_t bar0 = smem_u32(&bars[0]);
  auto bar = [&](int which, int i) { return bar0 + (uint32_t)(which + i) * 8u; };
  const volatile int* gu = &give_up;

  if (tid == 0) {
    for (int i = 0; i < p.slots; ++i) {
      mbar_init(bar(TB_FULL, i), TR_LOAD);                      // one arrival per loader warp
      mbar_init(bar(TB_EMPTY, i), 1);                           // a tcgen05.commit
    }
    for (int u = 0; u < 2; ++u) {
      mbar_init(bar(TB_S, u), 1);                               // a tcgen05.commit
      mbar_init(bar(TB_P, u), 4);                               // the group's warps
    }
    give_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (warp == TR_SOFT + TR_LOAD) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_base_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  chain_enter();
  // query rows t G + h of this group, zeros behind the last
  for (int i = tid; i < (p.two_rows ? 256 : 128) * (D / 8); i += TR_THREADS) {
    const int r = i / (D / 8), c = i % (D / 8), gr = row0 + r;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (r < rows) {
      v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + (((size_t)b * a.T + gr / G) * a.Hq + hk * G + gr % G) * D + c * 8);
      if (HALF) v = make_uint4(bf2_to_half2(v.x), bf2_to_half2(v.y), bf2_to_half2(v.z), bf2_to_half2(v.w));
    }
    sts128(sQ + (r >> 7) * SLOT + tile_off(r & 127, c), v);
  }
  asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem = tmem_base_slot;
  auto tS = [&](int u) { return tmem + (uint32_t)u * 128u; };
  auto tO = [&](int u) { return tmem + 256u + (uint32_t)u * D; };
  // stream u's tiles: all of them, or every second one
  auto stream_tiles = [&](int u) { return p.two_rows ? n_loc : (n_loc - u + 1) / 2; };

  float m_run = -INFINITY, l_run = 0.f;                         // softmax: this thread's row
  const float scale_log2 = 1.4426950408889634f * rsqrtf((float)D);

  if (warp < TR_SOFT) {
    // ---- softmax groups
    const int u = warp >> 2, rl = (warp & 3) * 32 + lane, r = (p.two_rows ? u * 128 : 0) + rl;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const bool work = (p.two_rows ? u * 128 : 0) + (warp & 3) * 32 < rows;      // warp-uniform: has rows
    const unsigned long long mask = r < rows ? a.mask[(size_t)b * a.T + (row0 + r) / G] & (~0ull >> (64 - a.T)) : 0ull;
    const int steps = stream_tiles(u);
    bool ok = true;
    for (int k = 0; k < steps; ++k) {
      const int j = j0 + (p.two_rows ? k : 2 * k + u);
      ok = mbar_wait(bar(TB_S, u), (uint32_t)(k & 1), gu);
      if (!ok) break;
      if (work) {
        asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
        const uint32_t ts = tS(u) + lanes;
        // which of 32 columns from c0 on this row sees
        auto visible = [&](int c0) -> uint32_t {
          const int lim = j < p.ctx_tiles ? a.n - 128 * j - c0 : a.n_tail - 128 * (j - p.ctx_tiles) - c0;
          uint32_t v = lim >= 32 ? 0xffffffffu : lim <= 0 ? 0u : (1u << lim) - 1u;
          if (j >= p.ctx_tiles && lim < 32) {                   // drafts: bit e of the mask is column lim + e
            const unsigned long long m = lim >= 0 ? mask << lim : lim > -64 ? mask >> -lim : 0ull;
            v |= (uint32_t)m;
          }
          return v;
        };
        const bool full = j < p.ctx_tiles && 128 * (j + 1) <= a.n;
        float mx = -INFINITY;
#pragma unroll 1
        for (int c0 = 0; c0 < 128; c0 += 64) {
          uint32_t x[32], y[32];
          tmem_ld32_issue(ts + c0, x);
          tmem_ld32_issue(ts + c0 + 32, y);
          tmem_wait(x);
          tmem_wait(y);
          if (full) {
#pragma unroll
            for (int i = 0; i < 32; ++i) mx = fmaxf(mx, fmaxf(__uint_as_float(x[i]), __uint_as_float(y[i])));
          } else {
            const uint32_t vx = visible(c0), vy = visible(c0 + 32);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              mx = fmaxf(mx, (vx >> i) & 1u ? __uint_as_float(x[i]) : -INFINITY);
              mx = fmaxf(mx, (vy >> i) & 1u ? __uint_as_float(y[i]) : -INFINITY);
            }
          }
          __syncwarp();
        }
        mx *= scale_log2;                                       // scale > 0; -inf stays
        // a new reference only where the old one is exceeded by more than 2^8 (or there is none yet)
        const bool renew = mx > m_run + 8.f;
        if (__any_sync(0xffffffffu, renew)) {
          const float mn = renew ? mx : m_run, corr = renew ? ex2a(m_run - mn) : 1.f;
          m_run = mn;
          l_run *= corr;
          if (k > 0) {
#pragma unroll 1
            for (int c0 = 0; c0 < D; c0 += 32) {
              uint32_t o[32];
              tmem_ld32_issue(tO(u) + lanes + c0, o);
              tmem_wait(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * corr);
              tmem_st32(tO(u) + lanes + c0, o);
            }
            tmem_wait_st();
          }
        }
        const float ref = m_run == -INFINITY ? 0.f : m_run;
        const uint64_t sc = pack2(scale_log2, scale_log2), nm = pack2(-ref, -ref);
        uint64_t sum2 = pack2(0.f, 0.f);
#pragma unroll 1
        for (int c0 = 0; c0 < 128; c0 += 32) {
          uint32_t x[32], pk[16];
          tmem_ld32_issue(ts + c0, x);
          tmem_wait(x);
          const uint32_t vis = full ? 0xffffffffu : visible(c0);
          if (!full) {
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = (vis >> i) & 1u ? x[i] : 0xff800000u;
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float e0, e1;
            unpack2(fma2(pack2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), sc, nm), e0, e1);
            e0 = ex2a(e0);
            e1 = ex2a(e1);
            sum2 = add2(sum2, pack2(e0, e1));
            if (HALF) {
              pk[i] = pack_half2(e0, e1);
            } else {
              const __nv_bfloat162 h = __floats2bfloat162_rn(e0, e1);
              pk[i] = *reinterpret_cast<const uint32_t*>(&h);
            }
          }
          __syncwarp();
          tmem_st16(ts + c0 / 2, pk);                           // over columns of S that have been read
        }
        float s0, s1;
        unpack2(sum2, s0, s1);
        l_run += s0 + s1;
        tmem_wait_st();
        asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(TB_P, u));
    }
    // O is complete with one more commit
    if (ok && steps > 0) {
      ok = mbar_wait(bar(TB_S, u), (uint32_t)(steps & 1), gu);
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    }
    if (!ok) give_up = 1;
  } else if (warp == TR_SOFT + TR_LOAD) {
    // ---- MMA warp.  Operand idx (keys of tile j: 2 j, values: 2 j + 1) sits in slot idx % slots.
    bool ok = true;
    auto wait_full = [&](int idx) { ok = ok && mbar_wait(bar(TB_FULL, idx % p.slots), (uint32_t)((idx / p.slots) & 1), gu); };
    auto issue_s = [&](int jl, int u, bool last_reader) {
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      if (lane == 0) {
        const uint32_t q = sQ + (p.two_rows ? u : 0) * SLOT, kk = ring + (2 * jl % p.slots) * SLOT;
#pragma unroll
        for (int kb = 0; kb < D / 64; ++kb)
#pragma unroll
          for (int s = 0; s < 4; ++s)
            umma_bf16(tS(u), smem_desc(q + kb * 16384 + s * 32), smem_desc(kk + kb * 16384 + s * 32), ID_S, (kb | s) ? 1u : 0u);
        if (last_reader) umma_commit(bar(TB_EMPTY, 2 * jl % p.slots));
        umma_commit(bar(TB_S, u));
      }
      __syncwarp();
    };
    auto issue_o = [&](int jl, int u, bool first, bool last_reader) {
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      if (lane == 0) {
        const uint32_t vv = ring + ((2 * jl + 1) % p.slots) * SLOT;
#pragma unroll
        for (int s = 0; s < 8; ++s)
          umma_ts(tO(u), tS(u) + 8 * s, smem_desc_mn(vv + s * 2048, 16384), ID_O, (first && s == 0) ? 0u : 1u);
        if (last_reader) umma_commit(bar(TB_EMPTY, (2 * jl + 1) % p.slots));
      }
      __syncwarp();
    };
    if (p.two_rows) {
      if (n_loc > 0) {
        wait_full(0);
        if (ok) issue_s(0, 0, false);
        if (ok) issue_s(0, 1, true);
      }
      for (int j = 0; j < n_loc && ok; ++j)
        for (int u = 0; u < 2 && ok; ++u) {
          if (u == 0) wait_full(2 * j + 1);
          ok = ok && mbar_wait(bar(TB_P, u), (uint32_t)(j & 1), gu);
          if (!ok) break;
          issue_o(j, u, j == 0, u == 1);
          if (j + 1 < n_loc) {
            if (u == 0) wait_full(2 * j + 2);
            if (ok) issue_s(j + 1, u, u == 1);
          } else {
            if (lane == 0) umma_commit(bar(TB_S, u));           // O[u] is complete
            __syncwarp();
          }
        }
    } else {
      for (int j = 0; j < min(2, n_loc) && ok; ++j) {
        wait_full(2 * j);
        if (ok) issue_s(j, j, true);
      }
      for (int j = 0; j < n_loc && ok; ++j) {
        const int u = j & 1;
        wait_full(2 * j + 1);
        ok = ok && mbar_wait(bar(TB_P, u), (uint32_t)((j >> 1) & 1), gu);
        if (!ok) break;
        issue_o(j, u, j < 2, true);
        if (j + 2 < n_loc) {
          wait_full(2 * j + 4);
          if (ok) issue_s(j + 2, u, true);
        } else {
          if (lane == 0) umma_commit(bar(TB_S, u));
          __syncwarp();
        }
      }
    }
    if (!ok) give_up = 1;
  } else {
    // ---- loader warps
    const int lt = tid - TR_SOFT * 32;
    bool ok = true;
    auto wait_empty = [&](int idx) {
      if (idx >= p.slots) ok = ok && mbar_wait(bar(TB_EMPTY, idx % p.slots), (uint32_t)((idx / p.slots - 1) & 1), gu);
    };
    auto slot_of = [&](int idx) { return ring + (idx % p.slots) * SLOT; };
    auto publish = [&](int idx) {                               // this warp's part of an operand is in place
      asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(TB_FULL, idx % p.slots));
    };
    const int n_ctx = max(0, min(n_loc, p.ctx_tiles - j0));     // this block's context tiles
    if constexpr (BITS == 16) {
      int issued = 0;
      for (int i = 0; i < 2 * n_ctx; ++i) {
        wait_empty(i);
        if (!ok) break;
        if (lane == 0) {
          if (warp == TR_SOFT) {
            mbar_expect_tx(bar(TB_FULL, i % p.slots), SLOT);
#pragma unroll
            for (int kb = 0; kb < D / 64; ++kb)
              tma_load_3d(slot_of(i) + kb * 16384, i & 1 ? &map_v : &map_k, kb * 64, 128 * (j0 + i / 2), bh, bar(TB_FULL, i % p.slots));
          } else {
            mbar_arrive(bar(TB_FULL, i % p.slots));
          }
        }
        issued = i + 1;
        __syncwarp();
      }
      if (!ok && warp == TR_SOFT) {
        // the copies still on their way land in this block's shared memory: wait (bounded) for them before it is given up
        for (int i = max(0, issued - p.slots); i < issued; ++i)
          for (uint32_t s = 0; s < TC_SPIN_LIMIT; ++s)
            if (mbar_try_wait(bar(TB_FULL, i % p.slots), (uint32_t)((i / p.slots) & 1))) break;
      }
    } else {
      RowLoader<BITS, D> rk, rv;
      ColLoader<BITS, D> ck;
      const bool cols = a.k_axis == 0;
      if (n_ctx > 0) {
        if (cols) ck.fetch(a, bh, 128 * j0, lt); else rk.fetch(a, a.kc, a.ks, a.kz, bh, 128 * j0, lt);
      }
      for (int j = 0; j < n_ctx && ok; ++j) {
        const int tok0 = 128 * (j0 + j);
        rv.fetch(a, a.vc, a.vs, a.vz, bh, tok0, lt);
        wait_empty(2 * j);
        if (!ok) break;
        if (cols) ck.put(a, tok0, lt, slot_of(2 * j)); else rk.put(a, tok0, lt, slot_of(2 * j));
        publish(2 * j);
        if (j + 1 < n_ctx) {
          if (cols) ck.fetch(a, bh, tok0 + 128, lt); else rk.fetch(a, a.kc, a.ks, a.kz, bh, tok0 + 128, lt);
        }
        wait_empty(2 * j + 1);
        if (!ok) break;
        rv.put(a, tok0, lt, slot_of(2 * j + 1));
        publish(2 * j + 1);
      }
    }
    for (int j = n_ctx; j < n_loc && ok; ++j)
      for (int kv = 0; kv < 2 && ok; ++kv) {
        wait_empty(2 * j + kv);
        if (!ok) break;
        put_extra<D, HALF>(a, kv == 0, b, hk, bh, j0 + j - p.ctx_tiles, lt, slot_of(2 * j + kv));
        publish(2 * j + kv);
      }
    if (!ok) give_up = 1;
  }

  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();                                              // every product is done: ring and queries are idle
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  constexpr uint32_t PART = 128 * D * 4;                        // one stream's O; the statistics [2][128] follow the two
  unsigned char* part_base = smem_raw + (sbase - smem_u32(smem_raw));
  float2* s_ml = reinterpret_cast<float2*>(part_base + 2 * PART);
  if (warp < TR_SOFT) {
    const int u = warp >> 2, rl = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const bool any = !give_up && stream_tiles(u) > 0 && (p.two_rows ? u * 128 : 0) + (warp & 3) * 32 < rows;
    s_ml[u * 128 + rl] = make_float2(any ? m_run : -INFINITY, l_run);
    if (any) {
#pragma unroll 1
      for (int c0 = 0; c0 < D; c0 += 32) {
        uint32_t o[32];
        tmem_ld32_issue(tO(u) + lanes + c0, o);
        tmem_wait(o);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          sts128(sbase + u * PART + part_off<D>(rl, c0 / 4 + i), make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]));
      }
    }
  }
  if (give_up && tid == 0) atomicExch(error_word, 1);
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  cluster.sync();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  if (warp == TR_SOFT + TR_LOAD)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512u) : "memory");

  // ---- this CTA's slice of the rows: a warp per row, lane c the contribution c (CTA c / per, stream c % per) for the
  // statistics, then the row's 16-byte chunk
  const int per = p.two_rows ? 1 : 2, n_part = C * per;         // <= 32
  const int r_lo = (int)((long long)rows * rank / C), r_hi = (int)((long long)rows * (rank + 1) / C);
  for (int r = r_lo + warp; r < r_hi; r += TR_THREADS / 32) {
    const int rl = r & 127, u_row = r >> 7;                     // two_rows: the stream that owns the row
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < n_part) ml = cluster.map_shared_rank(s_ml, lane / per)[(p.two_rows ? u_row : lane % per) * 128 + rl];
    float M = ml.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    const float f = ml.x == -INFINITY ? 0.f : ex2a(ml.x - M);
    float Z = ml.y * f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) Z += __shfl_xor_sync(0xffffffffu, Z, o);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = 0; c0 < n_part; c0 += 8) {
      float4 v[8];
      float fc[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        fc[i] = __shfl_sync(0xffffffffu, f, (c0 + i) & 31);
        const int c = c0 + i;
        v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < n_part && fc[i] != 0.f && lane < D / 4) {       // (a stream without tiles left nothing behind)
          const unsigned char* base = cluster.map_shared_rank(part_base, c / per);
          v[i] = *reinterpret_cast<const float4*>(base + (p.two_rows ? u_row : c % per) * PART + part_off<D>(rl, lane));
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        acc.x = fmaf(v[i].x, fc[i], acc.x); acc.y = fmaf(v[i].y, fc[i], acc.y);
        acc.z = fmaf(v[i].z, fc[i], acc.z); acc.w = fmaf(v[i].w, fc[i], acc.w);
      }
    }
    if (lane < D / 4) {
      const float inv = __fdiv_rn(1.0f, Z);
      const int gr = row0 + r;
      const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x * inv, acc.y * inv), hi = __floats2bfloat162_rn(acc.z * inv, acc.w * inv);
      *reinterpret_cast<uint2*>(static_cast<bf16*>(a.out) + (((size_t)b * a.T + gr / G) * a.Hq + hk * G + gr % G) * D + 4 * lane) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    }
  }
  cluster.sync();                                               // nobody leaves while another may still read its shared memory
}

// rows of one KV head as [n x D], zeros behind row n whatever the array holds there
cudaError_t token_map(CUtensorMap* map, const void* base, const TreeArgs& a) {
  EncodeTiledFn enc = encode_tiled();
  if (!enc) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {(cuuint64_t)a.D, (cuuint64_t)a.n, (cuuint64_t)a.Bt * a.Hkv};
  const cuuint64_t strides[2] = {(cuuint64_t)a.D * 2, (cuuint64_t)a.ns * a.D * 2};
  const cuuint32_t box[3] = {64, 128, 1}, elem[3] = {1, 1, 1};
  const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, elem,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int BITS, int D>
cudaError_t launch_tree_t(TreeLaunch p, const CUtensorMap& mk, const CUtensorMap& mv, int* err, cudaStream_t st) {
  static unsigned char done[64] = {};
  static int active[64][TR_MAX_CLUSTER + 1] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  constexpr size_t SLOT = 128 * (size_t)D * 2;
  constexpr size_t smem_max = 7 * SLOT + 1024;                  // queries and ring, or the partial results that overlay them
  auto kernel = tree_kernel<BITS, D>;
  e = allow_smem(kernel, smem_max, done);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(TR_THREADS);
  cfg.dynamicSmemBytes = smem_max;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  if (active[dev][0] == 0) {                                    // once per device: how many clusters of a size fit at once
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    for (int c = 1; c <= TR_MAX_CLUSTER; ++c) {
      int n = 0;
      cfg.gridDim = dim3(c);
      attr[0].val.clusterDim.x = c;
      cfg.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
      if (e != cudaSuccess) return e;
      active[dev][c] = n;
    }
    active[dev][0] = 1;
  }
  p.slots = p.two_rows ? 5 : 6;
  // CTAs per (KV head, row group): the shortest schedule, rounds of (tiles + about three tiles of set-up and exchange)
  const int items = p.a.Bt * p.a.Hkv * p.n_groups;
  double best = 1e300;
  p.cluster = 1;
  for (int c = 1; c <= TR_MAX_CLUSTER && c <= p.tiles; ++c) {
    if (active[dev][c] < 1) continue;
    const double cost = (double)((items + active[dev][c] - 1) / active[dev][c]) * ((p.tiles + c - 1) / c + 3);
    if (cost < best) { best = cost; p.cluster = c; }
  }
  cfg.gridDim = dim3((unsigned)items * p.cluster);
  attr[0].val.clusterDim.x = p.cluster;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, p, mk, mv, err);
}

}  // namespace

size_t tree_workspace(const TreeArgs&) { return 256; }

cudaError_t launch_tree(const TreeArgs& a, void* ws, cudaStream_t st) {
  int* err = reinterpret_cast<int*>(static_cast<char*>(ws) + tree_workspace(a) - 256);
  cudaError_t e = cudaMemsetAsync(err, 0, sizeof(int), st);
  if (e != cudaSuccess) return e;
  TreeLaunch p{};
  p.a = a;
  p.R = a.T * (a.Hq / a.Hkv);
  p.n_groups = (p.R + 255) / 256;
  p.two_rows = p.R > 128 ? 1 : 0;
  p.ctx_tiles = (a.n + 127) / 128;
  p.tiles = p.ctx_tiles + (a.n_tail + a.T + 127) / 128;
  CUtensorMap mk, mv;
  memset(&mk, 0, sizeof(mk));
  memset(&mv, 0, sizeof(mv));
  if (a.bits == 16) {
    e = token_map(&mk, a.kc, a);
    if (e == cudaSuccess) e = token_map(&mv, a.vc, a);
    if (e != cudaSuccess) return e;
  }
#define QP_TREE(BITS) return a.D == 128 ? launch_tree_t<BITS, 128>(p, mk, mv, err, st) : launch_tree_t<BITS, 64>(p, mk, mv, err, st)
  switch (a.bits) {
    case 2: QP_TREE(2);
    case 4: QP_TREE(4);
    case 8: QP_TREE(8);
    case 16: QP_TREE(16);
    default: return cudaErrorInvalidValue;
  }
#undef QP_TREE
}

}  // namespace qp
