// Attention of a tree of drafted tokens over a packed cache, its tail and the drafts themselves (qp_decode_attn_tree).
//
// The T drafts' G query heads of one KV head are R = T G rows of one attention problem over N = n + n_tail + T tokens: with
// 4 R D flop per token against 2 D B / 8 bytes of cache the tensor cores are as much the bound as HBM, so both products run on
// tcgen05, the codes are expanded to fp16 once per (KV head, tile) whatever R is, and all T drafts cost one pass over the cache.
//
// A block owns up to 256 rows of one KV head and walks over a run of 128-token tiles; its parts talk through mbarriers only:
//   loader warps      tile j -> keys, then values, into a ring of 32 KB operand slots (128-byte swizzle).  Packed caches: words,
//                     scales and zero points by asynchronous copies into raw stages, several operands ahead, then to fp16 and
//                     into the slot.  16-bit caches: TMA, with the token count as the tensor's extent, so rows behind the last
//                     one arrive as zeros whatever the array holds there.  Tail and drafts form the last one or two tiles.
//   1 MMA warp        S[u] = Q[u] K_j^T into tensor memory; O[u] += P[u] V_j with P from tensor memory and V read with its rows
//                     as the contraction, so neither operand is transposed
//   2 softmax groups  u = 0, 1, four warps each, one row per thread: no shuffles.  S is read twice (maximum; exponentials); P
//                     overwrites the columns of S already read.  O is rescaled only when the maximum grows by more than 2^8
//                     (the weights then stay below 2^8 in 16 bits, relative precision unchanged).
// u is a tile of 128 rows when there are two, else (R <= 128) the parity of the token tile: two independent streams either
// way, so one group's exponentials run beside the other's products.
//
// The runs of one (KV head, row group) form a cluster: partial (max, sum, O) stay in shared memory, every CTA adds up its slice
// of the rows from all of them through distributed shared memory and writes it.  Where clusters of the GPU's size would leave
// SMs idle, several smaller ones share a (KV head, row group) and a small kernel merges what they leave in the workspace.
// Order of additions fixed; every mbarrier wait bounded (see the score sweeps).
//
// Measured in a replayed graph (32 heads over 8): 8 drafts on 2048 tokens at 4 bit 12.0 us, mostly latencies one after another; 64
// on 8192 at 16 bit 26.9 us, of which the exchange of 128 KB per block (14 bytes a clock through distributed shared memory) is
// 4; 33 on 8 x 8192 at 2 bit 86 us = 0.41 PFLOP/s: a tile of two row tiles reads and writes 256 KB of shared memory at 128 bytes
// a clock, and the second row tile holds four rows.
//
// Types: 16-bit caches multiply in bf16; packed ones in fp16 (2^-11 on a reconstructed value, against 2^-8 in bf16), tail,
// drafts and queries converted (exact but for |x| below 2^-14, off by at most 2^-25, or above 65504).  Logits, maxima, sums
// and O in 32 bits; the softmax weights enter the second product in 16 bits like its values.
#include <cooperative_groups.h>

#include <algorithm>
#include <cstring>

#include "qp_cluster.cuh"
#include "qp_mma.cuh"
#include "qp_tc.cuh"

namespace qp {

namespace {

namespace cg = cooperative_groups;

constexpr int TR_SOFT = 8;                                       // softmax warps
// Loader warps: seven, so that with the MMA warp there are sixteen and every thread has 128 registers; with a seventeenth it is
// 96 and the softmax spills (8 x 8192 tokens, 33 drafts: 78 -> 104 us).  Softmax warps that have no rows load, too.
constexpr int TR_LOAD = 7;
// Teams of loaders: one expands the keys, one the values, each at its own pace (an operand is a chain of waits and barriers that
// one team after the other would walk).  At 8 bits there is no room for the raw stages of two.
__host__ __device__ constexpr int tr_teams(int bits) { return bits == 8 ? 1 : 2; }
constexpr int TR_THREADS = (TR_SOFT + TR_LOAD + 1) * 32;
constexpr int TR_MAX_SLOTS = 6, TR_MAX_CLUSTER = 16, TR_MAX_SUBS = 16;

enum : int { TB_FULL = 0, TB_EMPTY = TR_MAX_SLOTS, TB_S = 2 * TR_MAX_SLOTS, TB_P = TB_S + 2, TB_Q = TB_P + 2, TB_COUNT = TB_Q + 1 };

struct TreeLaunch {
  TreeArgs a;
  int R, n_groups;           // rows per KV head, groups of up to 256 of them
  int two_rows;              // 1: stream u = row tile u of the group; 0: stream u = parity of the token tile
  int ctx_tiles, tiles;      // context tiles, and with the tail's and drafts'
  int slots, raw;            // operand slots, raw stages (packed caches)
  int cluster, subs, max_subs;   // CTAs per cluster, clusters per (KV head, row group): more than one leave partial results
  int lg;                    // log2 of the quantization group
  int inv_g;                 // ceil(2^16 / G): a row below 512 times this, shifted by 16, is the row's draft
  float* part;               // [KV head, row group][sub][256][D], then
  float2* part_ml;           // [KV head, row group][sub][256]
};

// a place in a ring of n, with the parity of the round; walks without divisions
struct Ring {
  int i = 0;
  uint32_t round = 0;
  __device__ __forceinline__ void next(int n, int step = 1) {
    i += step;
    if (i >= n) { i -= n; round ^= 1u; }
  }
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
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(d) : "f"(a), "f"(b), "f"(c));
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

// ---- packed operands.  The words, scales and zero points of one operand (128 tokens of keys or of values) come into a raw stage
// by asynchronous copies, several operands ahead; then the loaders expand them into an operand slot.  Raw stage: codes, scales,
// zero points.  The codes of keys with groups along the tokens lie in rows of 8 channels (32 wpg bytes) with 16 bytes of pad, so
// that eight lanes with eight such rows hit different banks.
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
  unsigned short v;
  asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(v) : "r"(a));
  return v;
}
template <int BITS, int D>
struct Raw {
  static constexpr int CODES = 128 * D * BITS / 8 + (128 / 32) * (D / 8) * 16;  // most: groups of 32
  static constexpr int META = 128 * (D / 32) * 2;                               // of scales, or of zero points
  static constexpr int BYTES = CODES + 2 * META;
};
// Copies of one operand's valid tokens (a multiple of 32, of the group if the groups run along the tokens), tile after tile: the
// pointers walk.  lg: log2 of the group.
template <int BITS, int D>
struct RawCopy {
  const unsigned char *codes, *scale, *zero;                    // of the next tile, at this thread's first piece
  int lline;                                                    // log2 of the 16-byte pieces in a row of 8 channels; 31: no rows
  __device__ __forceinline__ void start(const void* c, const __half* s, const __half* z, size_t row, int lg, bool cols, int lt) {
    constexpr int LB = BITS == 8 ? 3 : BITS == 4 ? 2 : 1;
    codes = static_cast<const unsigned char*>(c) + row * (D * BITS / 8) + lt * 16;
    // scales and zero points: D/g a token row, or D a row of g tokens, either way row * D / g from the start
    scale = reinterpret_cast<const unsigned char*>(s) + (row * D >> lg) * 2 + lt * 16;
    zero = reinterpret_cast<const unsigned char*>(z) + (row * D >> lg) * 2 + lt * 16;
    lline = cols ? lg + LB - 4 : 31;
  }
  __device__ __forceinline__ void issue(int nt, int lg, int lt, int NT, uint32_t raw) {
    using R = Raw<BITS, D>;
    const int pieces = nt * (D * BITS / 8) / 16, meta = (nt * D >> lg) * 2 / 16;
    const unsigned char* c = codes;
    for (int i = lt; i < pieces; i += NT, c += NT * 16) cp_async16(raw + i * 16 + (i >> lline) * 16, c);
    for (int i = lt; i < meta; i += NT) {
      cp_async16(raw + R::CODES + i * 16, scale + (i - lt) * 16);
      cp_async16(raw + R::CODES + R::META + i * 16, zero + (i - lt) * 16);
    }
    codes += 128 * (D * BITS / 8);
    scale += (128 * D >> lg) * 2;
    zero += (128 * D >> lg) * 2;
  }
};
// Groups along the tokens (keys of the main path): an item is 8 channels x PT tokens, a word per channel.
template <int BITS, int D>
__device__ __forceinline__ void put_cols(const TreeArgs& a, int lg, int tok0, int lt, int NT, uint32_t raw, uint32_t slot) {
  using R = Raw<BITS, D>;
  constexpr int PER = 32 / BITS, PT = PER < 8 ? PER : 8, OCT = D / 8, ITEMS = (128 / PT) * OCT;
  const int g = 1 << lg, wpg = g * BITS / 32;
#pragma unroll 1
  for (int i = lt; i < ITEMS; i += NT) {
    const int oct = i % OCT, row = i / OCT * PT;
    if (tok0 + row >= a.n) {                                    // (n is a multiple of 32: an item is inside or outside)
#pragma unroll
      for (int e = 0; e < PT; ++e) sts128(slot + tile_off(row + e, oct), make_uint4(0u, 0u, 0u, 0u));
      continue;
    }
    const int u = row >> lg, e0 = row & (g - 1);
    const uint32_t src = raw + (u * OCT + oct) * (32 * wpg + 16) + e0 / PER * 4, m = raw + R::CODES + (u * D + oct * 8) * 2;
    uint32_t w[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) w[c] = lds32(src + c * wpg * 4);
    const uint4 sv = lds128(m), zv = lds128(m + R::META);
    const uint32_t s2[4] = {sv.x, sv.y, sv.z, sv.w}, z2[4] = {zv.x, zv.y, zv.z, zv.w};
    const bool upper = BITS == 2 && (e0 & 8);                   // 16 tokens a word, 8 an item
#pragma unroll
    for (int half = 0; half < (PT * BITS > 16 ? 2 : 1); ++half) {
      uint32_t x[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) x[c] = __byte_perm(w[2 * c], w[2 * c + 1], half || upper ? 0x7632 : 0x5410);
      constexpr int N = PT * BITS > 16 ? PT / 2 : PT;           // tokens in 16 bits
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
// Groups along the channels (values; keys quantized token by token): an item is 32 channels of one token.
template <int BITS, int D>
__device__ __forceinline__ void put_rows(const TreeArgs& a, int lg, int tok0, int lt, int NT, uint32_t raw, uint32_t slot) {
  using R = Raw<BITS, D>;
  constexpr int PIECES = D / 32, W = BITS;                      // words of an item
#pragma unroll 1
  for (int i = lt; i < 128 * PIECES; i += NT) {
    const int piece = i % PIECES, row = i / PIECES;
    // chunks 4 piece .. 4 piece + 3 of the row
    const uint32_t at = slot + (piece >> 1) * 16384 + (row >> 3) * 1024 + (row & 7) * 128;
    const uint32_t c0 = (piece & 1) * 4, sw = row & 7;
    if (tok0 + row >= a.n) {
#pragma unroll
      for (int q = 0; q < 4; ++q) sts128(at + (((c0 + q) ^ sw) << 4), make_uint4(0u, 0u, 0u, 0u));
      continue;
    }
    const uint32_t src = raw + (row * PIECES + piece) * (W * 4), m = raw + R::CODES + ((row * D + piece * 32) >> lg) * 2;
    const uint32_t s2 = lds16(m) * 0x10001u, z2 = lds16(m + R::META) * 0x10001u;
    uint32_t w[W];
    if constexpr (W == 2) {
      const uint2 x = lds64(src);
      w[0] = x.x; w[1] = x.y;
    } else {
#pragma unroll
      for (int j = 0; j < W; j += 4) {
        const uint4 x = lds128(src + j * 4);
        w[j] = x.x; w[j + 1] = x.y; w[j + 2] = x.z; w[j + 3] = x.w;
      }
    }
    // a word's pair f holds channels f and f + 16/BITS; pairs f, f + 1 make the channel pairs (f, f+1) and the upper ones
    constexpr int U = 16 / BITS;
    uint32_t c[16];                                             // channels (0,1) .. (30,31)
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int f = 0; f < U; f += 2) {
        const uint32_t p = code_pair<BITS>(w[j], f * BITS, s2, z2), q = code_pair<BITS>(w[j], (f + 1) * BITS, s2, z2);
        c[j * U + f / 2] = __byte_perm(p, q, 0x5410);
        c[j * U + U / 2 + f / 2] = __byte_perm(p, q, 0x7632);
      }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      sts128(at + (((c0 + q) ^ sw) << 4), make_uint4(c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]));
  }
}
// halves of w that are not finite (of fp16, or of bf16)
template <bool HALF>
__device__ __forceinline__ uint32_t not_finite2(uint32_t w) { return __vcmpgeu2(w & 0x7fff7fffu, HALF ? 0x7c007c00u : 0x7f807f80u); }

// rows 128 x .. of the tail followed by the drafts, zeros behind them.  A draft's value that is not finite must not reach the
// rows that do not see the draft (their weight 0 times it is NaN, and a padded tree may hold anything there): it becomes 0 and
// the draft's bit is set in `bad`; the rows that do see it get it at the end, see add_bad.
template <int D, bool HALF>
__device__ __forceinline__ void put_extra(const TreeArgs& a, bool keys, int b, int hk, int bh, int x, int lt, int NT, uint32_t slot,
                                          unsigned long long* bad) {
  constexpr int PIECES = D / 16;
  const uint16_t* tail = static_cast<const uint16_t*>(keys ? a.k_tail : a.v_tail);
  const uint16_t* draft = static_cast<const uint16_t*>(keys ? a.k_draft : a.v_draft);
#pragma unroll 2
  for (int i = lt; i < 128 * PIECES; i += NT) {
    const int piece = i % PIECES, row = i / PIECES, e = 128 * x + row;
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
      if (!keys && e >= a.n_tail) {
        uint32_t any = 0u;
        auto clear = [&](uint32_t& w) {
          const uint32_t m = not_finite2<HALF>(w);
          w &= ~m;
          any |= m;
        };
#pragma unroll
        for (int j = 0; j < 2; ++j) { clear(v[j].x); clear(v[j].y); clear(v[j].z); clear(v[j].w); }
        if (any) atomicOr(bad, 1ull << (e - a.n_tail));
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

// the values that put_extra left out, for row r of the partial O, which sees the drafts `hit` of them
template <int D, bool HALF>
__device__ __forceinline__ void add_bad(unsigned char* part, int r, unsigned long long hit, const uint16_t* draft, int stride) {
#pragma unroll 1
  for (; hit; hit &= hit - 1) {
    const uint16_t* v = draft + (size_t)(__ffsll((long long)hit) - 1) * stride;
#pragma unroll 1
    for (int d = 0; d < D; ++d) {
      const uint32_t w = HALF ? bf2_to_half2(v[d]) : v[d];
      if (not_finite2<HALF>(w) & 0xffffu) {
        float* o = reinterpret_cast<float*>(part + part_off<D>(r, d / 4)) + d % 4;
        *o += HALF ? __half2float(__ushort_as_half((unsigned short)w)) : __uint_as_float(w << 16);
      }
    }
  }
}

#ifdef QP_CHECKED
__device__ int g_give_up = -1;                                  // see qp_debug_give_up
#endif

template <int BITS, int D>
__global__ void __launch_bounds__(TR_THREADS, 1)
tree_kernel(const __grid_constant__ TreeLaunch p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
            int* __restrict__ error_words) {
  constexpr bool HALF = BITS < 16;
  constexpr int TEAMS = tr_teams(BITS);
  constexpr uint32_t SLOT = 128 * D * 2;
  constexpr uint32_t FMT = HALF ? 0u : (1u << 7) | (1u << 10);  // both operands fp16 / bf16
  constexpr uint32_t ID_S = (1u << 4) | FMT | ((128u >> 3) << 17) | ((128u >> 4) << 24);
  constexpr uint32_t ID_O = (1u << 4) | FMT | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);   // B: rows contract
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t bars[TB_COUNT];
  __shared__ uint32_t tmem_base_slot;
  __shared__ int give_up;
  __shared__ unsigned long long bad_drafts;                     // of this block's tiles: values that are not finite, see put_extra
  cg::cluster_group cluster = cg::this_cluster();

  const TreeArgs& a = p.a;
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int C = p.cluster, rank = blockIdx.x % C, sub = blockIdx.x / C % p.subs, item = blockIdx.x / C / p.subs;
  const int rg = item % p.n_groups, bh = item / p.n_groups;
  const int b = bh / a.Hkv, hk = bh % a.Hkv, G = a.Hq / a.Hkv;
  const int row0 = rg * 256, rows = min(256, p.R - row0);       // of this group
  const int run = sub * C + rank, runs = p.subs * C;
  const int j0 = (int)((long long)p.tiles * run / runs), n_loc = (int)((long long)p.tiles * (run + 1) / runs) - j0;
  // draft of row gr = t G + h of this KV head, and where its query or output row starts (t Hq + h = gr + t (Hq - G))
  const size_t q0 = ((size_t)b * a.T * a.Hq + hk * G) * D;
  auto draft_of = [&](int gr) { return (gr * p.inv_g) >> 16; };
  auto row_off = [&](int gr) { return q0 + (size_t)(gr + draft_of(gr) * (a.Hq - G)) * D; };
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sQ = sbase, ring = sbase + (p.two_rows ? 2 : 1) * SLOT;
  const uint32_t bar0 = smem_u32(&bars[0]);
  auto bar = [&](int which, int i) { return bar0 + (uint32_t)(which + i) * 8u; };
  const volatile int* gu = &give_up;

  // softmax warps at work: those with rows, and the first of each group; the others load.  Loaders are numbered from the
  // dedicated ones on, so that loader 0 is always warp TR_SOFT.
  auto warps_of = [&](int u) { return max(1, min(4, (rows - (p.two_rows ? u * 128 : 0) + 31) / 32)); };
  const int w0 = warps_of(0), w1 = warps_of(1), n_load = TR_LOAD + 8 - w0 - w1;
  // the keys' team: two fifths (their words come apart with less work); arrivals that fill an operand: the larger team
  const int k_load = TEAMS == 1 ? n_load : (2 * n_load + 2) / 5, full_load = max(k_load, n_load - k_load);
  const bool loads = warp < TR_SOFT ? (warp & 3) >= (warp < 4 ? w0 : w1) : warp < TR_SOFT + TR_LOAD;
  const int lw = warp >= TR_SOFT ? warp - TR_SOFT : TR_LOAD + (warp < 4 ? warp - w0 : 4 - w0 + (warp - 4) - w1);
  if (tid == 0) {
    for (int i = 0; i < p.slots; ++i) {
      mbar_init(bar(TB_FULL, i), full_load);                    // one arrival per warp of the larger team
      mbar_init(bar(TB_EMPTY, i), 1);                           // a tcgen05.commit
    }
    for (int u = 0; u < 2; ++u) {
      mbar_init(bar(TB_S, u), 1);                               // a tcgen05.commit
      mbar_init(bar(TB_P, u), u ? w1 : w0);                     // the group's warps at work
    }
    mbar_init(bar(TB_Q, 0), TR_SOFT);                           // the softmax warps, which fetch the queries
    give_up = 0;
    bad_drafts = 0ull;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (warp == TR_SOFT + TR_LOAD) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_base_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem = tmem_base_slot;
  chain_enter();                                                // the launch's set-up overlaps the previous kernel's end
  auto tS = [&](int u) { return tmem + (uint32_t)u * 128u; };
  auto tO = [&](int u) { return tmem + 256u + (uint32_t)u * D; };
  // stream u's tiles: all of them, or every second one
  auto stream_tiles = [&](int u) { return p.two_rows ? n_loc : (n_loc - u + 1) / 2; };

  float m_run = -INFINITY, l_run = 0.f;                         // softmax: this thread's row
  const float scale_log2 = 1.4426950408889634f * rsqrtf((float)D);

  if (warp < TR_SOFT) {
    // the first eight warps fetch the query rows t G + h of this group, zeros behind the last, eight loads in flight
    for (int i0 = tid; i0 < (p.two_rows ? 256 : 128) * (D / 8); i0 += 8 * TR_SOFT * 32) {
      uint4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = i0 + k * TR_SOFT * 32, r = i / (D / 8), c = i % (D / 8), gr = row0 + r;
        v[k] = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows)
          v[k] = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + row_off(gr) + c * 8));
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = i0 + k * TR_SOFT * 32, r = i / (D / 8), c = i % (D / 8);
        if (HALF) v[k] = make_uint4(bf2_to_half2(v[k].x), bf2_to_half2(v[k].y), bf2_to_half2(v[k].z), bf2_to_half2(v[k].w));
        if (r < (p.two_rows ? 256 : 128)) sts128(sQ + (r >> 7) * SLOT + tile_off(r & 127, c), v[k]);
      }
    }
    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(TB_Q, 0));
  }

  if (warp < TR_SOFT && !loads) {
    // ---- softmax groups
    const int u = warp >> 2, rl = (warp & 3) * 32 + lane, r = (p.two_rows ? u * 128 : 0) + rl;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const bool work = (p.two_rows ? u * 128 : 0) + (warp & 3) * 32 < rows;      // warp-uniform: has rows
    const unsigned long long mask = r < rows ? a.mask[(size_t)b * a.T + draft_of(row0 + r)] & (~0ull >> (64 - a.T)) : 0ull;
    const int steps = stream_tiles(u);                          // (a group without rows has its first warp here to answer for it)
    bool ok = true;
    for (int k = 0; k < steps; ++k) {
      const int j = j0 + (p.two_rows ? k : 2 * k + u);
      ok = mbar_wait_warp(bar(TB_S, u), (uint32_t)(k & 1), gu);
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
        if (!full) {                                            // what the row does not see leaves S
#pragma unroll 1
          for (int c0 = 0; c0 < 128; c0 += 16) {
            const uint32_t vis = visible(c0 & ~31) >> (c0 & 16);
            uint32_t x[16];
            tmem_ld16_issue(ts + c0, x);
            tmem_wait16(x);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = (vis >> i) & 1u ? x[i] : 0xff800000u;
            __syncwarp();
            tmem_st(ts + c0, x);
          }
          tmem_wait_st();
        }
        // (loops, not unrolled: the kernel waits for instructions otherwise; the loaders' unrolled by two cost 20 %)
        uint32_t xa[32], xb[32];
        float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll 1
        for (int c0 = 0; c0 < 128; c0 += 64) {
          tmem_ld32_issue(ts + c0, xa);
          tmem_ld32_issue(ts + c0 + 32, xb);
          tmem_wait(xa);
          tmem_wait(xb);
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            mx0 = max3(mx0, __uint_as_float(xa[i]), __uint_as_float(xa[i + 1]));
            mx1 = max3(mx1, __uint_as_float(xb[i]), __uint_as_float(xb[i + 1]));
          }
        }
        const float mx = fmaxf(mx0, mx1) * scale_log2;          // scale > 0; -inf stays
        // a new reference only where the old one is exceeded by more than 2^8 (or there is none yet)
        const bool renew = mx > m_run + 8.f;
        if (__any_sync(0xffffffffu, renew)) {
          const float mn = renew ? mx : m_run, corr = renew ? ex2a(m_run - mn) : 1.f;
          m_run = mn;
          l_run *= corr;
          if (k > 0) {
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {
              uint32_t o[16];
              tmem_ld16_issue(tO(u) + lanes + c, o);
              tmem_wait16(o);
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * corr);
              __syncwarp();
              tmem_st(tO(u) + lanes + c, o);
            }
            tmem_wait_st();
          }
        }
        // A reference that lags leaves a heavy weight a number that bf16 rounds by up to 2^-8: the sum takes the rounded weights, so
        // that the output stays a mean of the values and the heavy one's rounding cancels (2 drafts on 4484 tokens at 16 bit: error
        // of the output 0.0030 -> 0.0024; 64 on 8192: 0.0022 -> 0.0021, and 24.4 us with or without).  In fp16 it is 2^-11, below
        // what the output's own rounding shows.
        const float ref = m_run == -INFINITY ? 0.f : m_run;
        const uint64_t sc = pack2(scale_log2, scale_log2), nm = pack2(-ref, -ref);
        uint64_t sum2 = pack2(0.f, 0.f), sum3 = sum2;
        // 32 columns: P over columns of S that have been read
        auto fold = [&](const uint32_t (&x)[32], int c0) {
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float e0, e1;
            unpack2(fma2(pack2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), sc, nm), e0, e1);
            e0 = ex2a(e0);
            e1 = ex2a(e1);
            pk[i] = HALF ? pack_half2(e0, e1) : pack_bf16x2(e0, e1);
            if (!HALF) {                                        // the sum is of the weights as the product has them: see above
              e0 = bf16lo(pk[i]);
              e1 = bf16hi(pk[i]);
            }
            if (i & 1) sum3 = add2(sum3, pack2(e0, e1)); else sum2 = add2(sum2, pack2(e0, e1));
          }
          __syncwarp();
          tmem_st(ts + c0 / 2, pk);
        };
        tmem_ld32_issue(ts, xa);
#pragma unroll 1
        for (int c0 = 0; c0 < 128; c0 += 64) {
          tmem_wait(xa);
          tmem_ld32_issue(ts + c0 + 32, xb);
          fold(xa, c0);
          tmem_wait(xb);
          if (c0 == 0) tmem_ld32_issue(ts + 64, xa);
          fold(xb, c0 + 32);
        }
        sum2 = add2(sum2, sum3);
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
      ok = mbar_wait_warp(bar(TB_S, u), (uint32_t)(steps & 1), gu);
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    }
    if (!ok) give_up = 1;
  } else if (!loads) {
    // ---- MMA warp.  Operands in the ring: keys of tile 0, values of tile 0, keys of tile 1, ...
    bool ok = true;
    Ring kr, vr;                                                // the next keys and values
    vr.next(p.slots);
    auto wait_full = [&](const Ring& r) { ok = ok && mbar_wait_warp(bar(TB_FULL, r.i), r.round, gu); };
    auto issue_s = [&](int u, bool last_reader) {
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      const uint32_t q = uniform(desc_lo(sQ + (p.two_rows ? u : 0) * SLOT, 1)), kk = uniform(desc_lo(ring + kr.i * SLOT, 1));
      const uint32_t d = uniform(tS(u)), done = uniform(bar(TB_S, u)), empty = uniform(bar(TB_EMPTY, kr.i));
      if (elect_one()) {
        umma_ss<false>(d, q, kk, ID_S);
#pragma unroll
        for (int s = 1; s < D / 16; ++s) umma_ss<true>(d, q + (s / 4) * 1024 + (s % 4) * 2, kk + (s / 4) * 1024 + (s % 4) * 2, ID_S);
        umma_commit(done);
        if (last_reader) umma_commit(empty);
      }
      __syncwarp();
      if (last_reader) kr.next(p.slots, 2);
    };
    auto issue_o = [&](int u, bool first, bool last_reader) {
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      // values with their rows as the contraction: blocks of 64 columns are 16 KB apart, 16 rows 2 KB
      const uint32_t vv = uniform(desc_lo(ring + vr.i * SLOT, 1024)), d = uniform(tO(u)), pp = uniform(tS(u));
      const uint32_t empty = uniform(bar(TB_EMPTY, vr.i));
      if (elect_one()) {
        umma_ts(d, pp, vv, ID_O, first ? 0u : 1u);
#pragma unroll
        for (int s = 1; s < 8; ++s) umma_ts(d, pp + 8 * s, vv + s * 128, ID_O, 1u);
        if (last_reader) umma_commit(empty);
      }
      __syncwarp();
      if (last_reader) vr.next(p.slots, 2);
    };
    // stream u's last product is followed by one more commit: O[u] is complete
    auto finish = [&](int u) {
      const uint32_t done = uniform(bar(TB_S, u));
      if (elect_one()) umma_commit(done);
      __syncwarp();
    };
    ok = mbar_wait_warp(bar(TB_Q, 0), 0u, gu);
    if (p.two_rows) {
      if (n_loc > 0) {
        wait_full(kr);
        if (ok) issue_s(0, false);
        if (ok) issue_s(1, true);
      }
      for (int j = 0; j < n_loc && ok; ++j)
        for (int u = 0; u < 2 && ok; ++u) {
          if (u == 0) wait_full(vr);
          ok = ok && mbar_wait_warp(bar(TB_P, u), (uint32_t)(j & 1), gu);
          if (!ok) break;
          issue_o(u, j == 0, u == 1);
          if (j + 1 < n_loc) {
            if (u == 0) wait_full(kr);
            if (ok) issue_s(u, u == 1);
          } else {
            finish(u);
          }
        }
    } else {
      for (int j = 0; j < min(2, n_loc) && ok; ++j) {
        wait_full(kr);
        if (ok) issue_s(j, true);
      }
      for (int j = 0; j < n_loc && ok; ++j) {
        const int u = j & 1;
        wait_full(vr);
        ok = ok && mbar_wait_warp(bar(TB_P, u), (uint32_t)((j >> 1) & 1), gu);
        if (!ok) break;
        issue_o(u, j < 2, true);
        if (j + 2 < n_loc) {
          wait_full(kr);
          if (ok) issue_s(u, true);
        } else {
          finish(u);
        }
      }
    }
    if (!ok) give_up = 1;
  } else {
    // ---- loader warps
    const int team = TEAMS == 2 && lw >= k_load ? 1 : 0, t_size = TEAMS == 1 ? n_load : team ? n_load - k_load : k_load;
    const int tw = lw - (team ? k_load : 0), NT = t_size * 32, lt = tw * 32 + lane;
    const bool first = tw == 0;                                 // the team's first warp also arrives for those that a smaller team lacks
    const uint32_t arrivals = first ? 1 + full_load - t_size : 1;
    // operand i: keys (even) or values (odd) of this block's tile i / 2; this team's are team, team + TEAMS, ...
    bool ok = true;
    Ring wr;                                                    // the team's next operand's slot
    if (team) wr.next(p.slots);
    auto wait_empty = [&](int i) {
      if (i >= p.slots) ok = ok && mbar_wait_warp(bar(TB_EMPTY, wr.i), wr.round ^ 1u, gu);
    };
    auto slot = [&]() { return ring + wr.i * SLOT; };
    auto publish = [&]() {                                      // this warp's part of an operand is in place
      asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive_n(bar(TB_FULL, wr.i), arrivals);
      wr.next(p.slots, TEAMS);
    };
    const int n_ctx = max(0, min(n_loc, p.ctx_tiles - j0));     // this block's context tiles
    int i = team;
    if constexpr (BITS == 16) {
      // one lane of the team copies; the others follow the ring, whose parity they could not tell after two rounds
      Ring back = wr;                                           // the oldest copy that may still be on its way
      int flying = 0;
      for (; i < 2 * n_ctx; i += TEAMS) {
        wait_empty(i);
        if (i == team + TEAMS) ok = ok && mbar_wait_warp(bar(TB_Q, 0), 0u, gu);   // the queries overtake all but the first tile
        if (!ok) break;
        if (first && lane == 0) {
          mbar_expect_tx(bar(TB_FULL, wr.i), SLOT);
#pragma unroll
          for (int kb = 0; kb < D / 64; ++kb)
            tma_load_3d(slot() + kb * 16384, team ? &map_v : &map_k, kb * 64, 128 * (j0 + i / 2), bh, bar(TB_FULL, wr.i));
          mbar_arrive_n(bar(TB_FULL, wr.i), full_load - 1);
        }
        __syncwarp();
        wr.next(p.slots, TEAMS);
        if (flying == p.slots) back.next(p.slots, TEAMS); else ++flying;
      }
      if (!ok && first)
        // the copies still on their way land in this block's shared memory: wait (bounded) for them before it is given up
        for (; flying > 0; --flying, back.next(p.slots, TEAMS))
          for (uint32_t s = 0; s < TC_SPIN_LIMIT; ++s)
            if (mbar_try_wait(bar(TB_FULL, back.i), back.round)) break;
    } else {
      const bool cols = a.k_axis == 0;
      const int stages = p.raw / TEAMS;
      const uint32_t raw0 = ring + p.slots * SLOT + team * stages * Raw<BITS, D>::BYTES, raw_end = raw0 + stages * Raw<BITS, D>::BYTES;
      uint32_t raw_in = raw0, raw_out = raw0;
      RawCopy<BITS, D> ck, cv;                                  // a team of two uses one of them
      const size_t row0_ctx = (size_t)bh * a.ns + 128 * j0;
      if (TEAMS == 1 || team == 0) ck.start(a.kc, a.ks, a.kz, row0_ctx, p.lg, cols, lt);
      if (TEAMS == 1) cv.start(a.vc, a.vs, a.vz, row0_ctx, p.lg, false, lt);
      else if (team == 1) ck.start(a.vc, a.vs, a.vz, row0_ctx, p.lg, false, lt);
      auto issue = [&](int op) {
        if (op < 2 * n_ctx) {
          const int nt = min(128, a.n - 128 * (j0 + op / 2));
          if (TEAMS == 1 && (op & 1)) cv.issue(nt, p.lg, lt, NT, raw_in);
          else ck.issue(nt, p.lg, lt, NT, raw_in);
        }
        cp_async_commit();
        raw_in += Raw<BITS, D>::BYTES;
        if (raw_in == raw_end) raw_in = raw0;
      };
      for (int k = 0; k < stages - 1; ++k) issue(team + k * TEAMS);
      for (; i < 2 * n_ctx; i += TEAMS) {
        if (stages == 2) cp_async_wait<0>(); else if (stages == 3) cp_async_wait<1>(); else cp_async_wait<2>();   // this thread's part
        asm volatile("bar.sync %0, %1;\n" ::"r"(1 + team), "r"(NT) : "memory");     // the team's; and the stage before is used up
        issue(i + (stages - 1) * TEAMS);
        wait_empty(i);
        if (ok) {                                               // (otherwise keep the team's barrier together)
          const int tok0 = 128 * (j0 + i / 2);
          if (cols && !(i & 1)) put_cols<BITS, D>(a, p.lg, tok0, lt, NT, raw_out, slot());
          else put_rows<BITS, D>(a, p.lg, tok0, lt, NT, raw_out, slot());
          publish();
        }
        raw_out += Raw<BITS, D>::BYTES;
        if (raw_out == raw_end) raw_out = raw0;
      }
      cp_async_wait<0>();
    }
    for (; i < 2 * n_loc && ok; i += TEAMS) {
      wait_empty(i);
      if (!ok) break;
      put_extra<D, HALF>(a, !(i & 1), b, hk, bh, j0 + i / 2 - p.ctx_tiles, lt, NT, slot(), &bad_drafts);
      publish();
    }
    if (!ok) give_up = 1;
  }

  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();                                              // every product is done: ring and queries are idle
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#ifdef QP_CHECKED
  if (tid == 0 && (int)blockIdx.x == g_give_up) give_up = 1;    // (every wait of the block has returned)
  __syncthreads();
#endif
  constexpr uint32_t PART = 128 * D * 4;                        // one stream's O; the statistics [2][128] follow the two
  unsigned char* part_base = smem_raw + (sbase - smem_u32(smem_raw));
  float2* s_ml = reinterpret_cast<float2*>(part_base + 2 * PART);
  if (warp < TR_SOFT) {
    const int u = warp >> 2, rl = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const bool any = !give_up && stream_tiles(u) > 0 && (p.two_rows ? u * 128 : 0) + (warp & 3) * 32 < rows;
    // What the block lost, because a wait ran out, must not look like a run in which nothing was seen: with a reference that counts
    // and a sum that is no number the row's output is NaN, whatever the partial O holds.
    s_ml[u * 128 + rl] = give_up ? make_float2(0.f, NAN) : make_float2(any ? m_run : -INFINITY, l_run);
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
      const int r = (p.two_rows ? u * 128 : 0) + rl;
      if (bad_drafts && r < rows) {
        unsigned long long hit = bad_drafts & a.mask[(size_t)b * a.T + draft_of(row0 + r)];
        if (!p.two_rows) {                                      // this stream's part of a row: the drafts of every second tile
          const unsigned long long first = a.n_tail + a.T <= 128 ? ~0ull : (1ull << (128 - a.n_tail)) - 1;   // of the first extra tile
          hit &= ((p.ctx_tiles - j0) & 1) == u ? first : ~first;
        }
        add_bad<D, HALF>(part_base + u * PART, rl, hit, static_cast<const uint16_t*>(a.v_draft) + ((size_t)b * a.T * a.Hkv + hk) * D,
                         a.Hkv * D);
      }
    }
  }
  const int word = item * p.max_subs + sub;
  if (tid == 0 && rank == 0) {                                  // (the cluster's barrier orders it before the next)
    error_words[word] = 0;
    for (int s = p.subs; sub == 0 && s < p.max_subs; ++s) error_words[item * p.max_subs + s] = 0;
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  cluster.sync();
  if (give_up && tid == 0) atomicExch(&error_words[word], 1);
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  if (warp == TR_SOFT + TR_LOAD)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512u) : "memory");

  // ---- this CTA's slice of the rows.  Contribution c of a row is with CTA c (two row tiles; the row's stream), or with CTA c / 2,
  // stream c % 2
  const int sh = p.two_rows ? 0 : 1, n_part = C << sh;          // <= 32
  const int r_lo = (int)((long long)rows * rank / C), n_rows = (int)((long long)rows * (rank + 1) / C) - r_lo;
  // their statistics, n_rows * n_part <= 256 + 32 pairs, behind this CTA's own
  float2* s_all = s_ml + 256;
  for (int i = tid; i < n_rows * n_part; i += TR_THREADS) {
    const int r = r_lo + i / n_part, c = i % n_part;
    s_all[i] = cluster.map_shared_rank(s_ml, c >> sh)[(p.two_rows ? r >> 7 : c & 1) * 128 + (r & 127)];
  }
  __syncthreads();
  // a unit is a 16-byte chunk of a row's output; a remote read takes about a microsecond, so a thread has eight in flight: of
  // four units from two CTAs each where it has several units, sixteen of one unit else
  auto emit = [&](int r, int ch, float M, float Z, float4 acc) {
    if (p.subs > 1) {                                           // for the merge: unnormalised, with its reference and sum
      const size_t row = ((size_t)item * p.subs + sub) * 256 + r;
      *reinterpret_cast<float4*>(p.part + row * D + 4 * ch) = acc;
      if (ch == 0) p.part_ml[row] = make_float2(M, Z);
    } else {
      const float inv = __fdiv_rn(1.0f, Z);
      *reinterpret_cast<uint2*>(static_cast<bf16*>(a.out) + row_off(row0 + r) + 4 * ch) =
          make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    }
  };
  auto fetch = [&](int r, int ch, int c, float2 ml) {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (ml.x != -INFINITY)                                      // (a stream without tiles left nothing behind)
      v = *reinterpret_cast<const float4*>(cluster.map_shared_rank(part_base, c >> sh) + (p.two_rows ? r >> 7 : c & 1) * PART +
                                           part_off<D>(r & 127, ch));
    return v;
  };
  auto fold_in = [&](float4& acc, float& Z, float M, float2 ml, float4 v) {
    const float f = ml.x == -INFINITY ? 0.f : ex2a(ml.x - M);
    Z = fmaf(ml.y, f, Z);
    acc.x = fmaf(v.x, f, acc.x); acc.y = fmaf(v.y, f, acc.y);
    acc.z = fmaf(v.z, f, acc.z); acc.w = fmaf(v.w, f, acc.w);
  };
  const int units = n_rows * (D / 4);
  const float2 none = make_float2(-INFINITY, 0.f);
  if (units > TR_THREADS) {
    for (int i0 = tid; i0 < units; i0 += 4 * TR_THREADS) {
      float4 acc[4];
      float M[4], Z[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = i0 + k * TR_THREADS;
        M[k] = -INFINITY;
        Z[k] = 0.f;
        acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < units)
          for (int c = 0; c < n_part; ++c) M[k] = fmaxf(M[k], s_all[i / (D / 4) * n_part + c].x);
      }
      for (int c0 = 0; c0 < n_part; c0 += 2) {
        float4 v[4][2];
        float2 ml[4][2];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int i = i0 + k * TR_THREADS, rr = i / (D / 4);
            ml[k][j] = i < units && c0 + j < n_part ? s_all[rr * n_part + c0 + j] : none;
            v[k][j] = fetch(r_lo + rr, i % (D / 4), c0 + j, ml[k][j]);
          }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int j = 0; j < 2; ++j) fold_in(acc[k], Z[k], M[k], ml[k][j], v[k][j]);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = i0 + k * TR_THREADS;
        if (i < units) emit(r_lo + i / (D / 4), i % (D / 4), M[k], Z[k], acc[k]);
      }
    }
  } else if (tid < units) {
    const int rr = tid / (D / 4), ch = tid % (D / 4), r = r_lo + rr;
    float M = -INFINITY, Z = 0.f;
    for (int c = 0; c < n_part; ++c) M = fmaxf(M, s_all[rr * n_part + c].x);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = 0; c0 < n_part; c0 += 16) {
      float4 v[16];
      float2 ml[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        ml[k] = c0 + k < n_part ? s_all[rr * n_part + c0 + k] : none;
        v[k] = fetch(r, ch, c0 + k, ml[k]);
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) fold_in(acc, Z, M, ml[k], v[k]);
    }
    emit(r, ch, M, Z, acc);
  }
  cluster.sync();                                               // nobody leaves while another may still read its shared memory
}

// out from the partial results of several clusters per (KV head, row group), in their order: a 16-byte chunk of a row per thread
template <int D>
__global__ void __launch_bounds__(256)
tree_merge_kernel(const __grid_constant__ TreeLaunch p) {
  chain_enter();
  const TreeArgs& a = p.a;
  const int item = blockIdx.y, rg = item % p.n_groups, bh = item / p.n_groups, b = bh / a.Hkv, hk = bh % a.Hkv, G = a.Hq / a.Hkv;
  const int i = blockIdx.x * 256 + threadIdx.x, r = i / (D / 4), ch = i % (D / 4), gr = rg * 256 + r;
  if (gr >= p.R || r >= 256) return;
  const size_t row = (size_t)item * p.subs * 256 + r;
  float2 ml[TR_MAX_SUBS];
  float4 v[TR_MAX_SUBS];
  float M = -INFINITY, Z = 0.f;
#pragma unroll
  for (int s = 0; s < TR_MAX_SUBS; ++s)
    if (s < p.subs) {
      ml[s] = p.part_ml[row + s * 256];
      v[s] = *reinterpret_cast<const float4*>(p.part + (row + s * 256) * D + 4 * ch);
    }
#pragma unroll
  for (int s = 0; s < TR_MAX_SUBS; ++s)
    if (s < p.subs) M = fmaxf(M, ml[s].x);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int s = 0; s < TR_MAX_SUBS; ++s)
    if (s < p.subs && ml[s].x != -INFINITY) {                   // (-inf: a run in which the row sees nothing)
      const float f = ex2a(ml[s].x - M);
      Z = fmaf(ml[s].y, f, Z);
      acc.x = fmaf(v[s].x, f, acc.x); acc.y = fmaf(v[s].y, f, acc.y);
      acc.z = fmaf(v[s].z, f, acc.z); acc.w = fmaf(v[s].w, f, acc.w);
    }
  const float inv = __fdiv_rn(1.0f, Z);
  *reinterpret_cast<uint2*>(static_cast<bf16*>(a.out) + (((size_t)b * a.T + gr / G) * a.Hq + hk * G + gr % G) * D + 4 * ch) =
      make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
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

// most clusters per (KV head, row group): as many as keep every SM busy with clusters of one.  A B200's 148 and not the device's
// count, because the layout of the workspace, which the interface gives, goes by it.
int tree_max_subs(int items) { return std::max(1, std::min(TR_MAX_SUBS, 148 / items)); }
struct TreeWorkspace {
  size_t part, part_ml, total;   // the error words come first
};
TreeWorkspace tree_carve(const TreeArgs& a) {
  const int items = a.Bt * a.Hkv * ((a.T * (a.Hq / a.Hkv) + 255) / 256), subs = tree_max_subs(items);
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  TreeWorkspace w;
  w.part = up((size_t)items * subs * sizeof(int));
  w.part_ml = w.part + (subs > 1 ? (size_t)items * subs * 256 * a.D * sizeof(float) : 0);
  w.total = w.part_ml + (subs > 1 ? (size_t)items * subs * 256 * sizeof(float2) : 0);
  return w;
}

template <int BITS, int D>
cudaError_t launch_tree_t(TreeLaunch p, const CUtensorMap& mk, const CUtensorMap& mv, int* err, cudaStream_t st) {
  static int active[64][TR_MAX_CLUSTER + 1] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  constexpr size_t SLOT = 128 * (size_t)D * 2;
  constexpr size_t smem_max = 7 * SLOT + 1024;                  // queries and ring, or the partial results that overlay them
  auto kernel = tree_kernel<BITS, D>;
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
  e = clusters_that_fit(kernel, cfg, TR_MAX_CLUSTER, active[dev]);
  if (e != cudaSuccess) return e;
  if (BITS == 16) {
    p.slots = p.two_rows ? 5 : 6;
  } else {                                                      // the least the order of the products needs; raw stages from the rest
    p.slots = p.two_rows ? 3 : 4;
    p.raw = std::min(8, (int)(2 * SLOT / Raw<BITS == 16 ? 8 : BITS, D>::BYTES)) / tr_teams(BITS) * tr_teams(BITS);   // 3, 4 or 8
  }
  // CTAs per cluster and clusters per (KV head, row group): the shortest schedule, rounds of (tiles + about three tiles of set-up
  // and exchange), the merge of several clusters about another one and a half.  Large clusters need no merge, but leave SMs idle
  // that do not fill one inside their GPC.
  const int items = p.a.Bt * p.a.Hkv * p.n_groups, max_subs = tree_max_subs(items);
  double best = 1e300;
  p.cluster = p.subs = 1;
  p.max_subs = max_subs;
  for (int c = 1; c <= TR_MAX_CLUSTER && c <= p.tiles; ++c) {
    if (active[dev][c] < 1) continue;
    for (int s = 1; s <= max_subs && s * c <= p.tiles; ++s) {
      const double cost = (double)(((long long)items * s + active[dev][c] - 1) / active[dev][c]) * ((p.tiles + s * c - 1) / (s * c) + 3) +
                          (s > 1 ? 1.5 : 0.) + 0.01 * c;
      if (cost < best) { best = cost; p.cluster = c; p.subs = s; }
    }
  }
  cfg.gridDim = dim3((unsigned)items * p.subs * p.cluster);
  attr[0].val.clusterDim.x = p.cluster;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, kernel, p, mk, mv, err);
  if (e != cudaSuccess || p.subs == 1) return e;
  const int chunks = std::min(256, p.R) * (D / 4);
  return launch_chained(tree_merge_kernel<D>, dim3((chunks + 255) / 256, items), dim3(256), 0, st, p);
}

}  // namespace

size_t tree_workspace(const TreeArgs& a) { return tree_carve(a).total; }

#ifdef QP_CHECKED
cudaError_t tree_give_up(int block) { return cudaMemcpyToSymbol(g_give_up, &block, sizeof(block)); }
#endif

cudaError_t launch_tree(const TreeArgs& a, void* ws, cudaStream_t st) {
  int* err = static_cast<int*>(ws);
  cudaError_t e = cudaSuccess;
  TreeLaunch p{};
  const TreeWorkspace w = tree_carve(a);
  p.part = reinterpret_cast<float*>(static_cast<char*>(ws) + w.part);
  p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + w.part_ml);
  p.inv_g = (65536 + a.Hq / a.Hkv - 1) / (a.Hq / a.Hkv);
  p.lg = a.group == 32 ? 5 : a.group == 64 ? 6 : 7;
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
