// Attention of a step's new tokens over a paged cache in 8 bits (qp_paged_attn): many rows per KV head, as a prompt's chunk has.
//
// The G n query rows of a KV head are one attention problem of 4 G n D flop a token, far above what the cache's bytes cost, so both
// products run on tcgen05: S = Q K^T from shared memory, O += P V with P from tensor memory.  The codes are turned into fp16
// operands in shared memory once for 256 rows.
//   e4m3   by the hardware's conversion; int8: with the codes as low bits of 1024 + 128 + c.  Neighbouring int8 codes of a word come
//          out as channels (0, 2) and (1, 3), so operands hold the channels of every four in the order 0, 2, 1, 3: the queries are
//          stored in the same order, and the output's columns are put right when they leave.
// The scale of a page's keys multiplies 32 columns of S at a time; that of its values enters the exponent of their weights:
// P = 2^(x + log2(scale) - M) with M the running maximum of that sum, and the row's sum takes P s0 / scale, in 32 bits, s0 being the
// scale at the beginning of what the block does of the item: good for pages whose scales are within 2^90 of one another.
//
// Work: an item is (sequence, 256 rows, KV head); its tiles are the 128-token pieces of what its last row sees.  All items' tiles form
// one sequence (a small kernel numbers them, from the lengths on the device), cut into one equal run for each of 148 blocks.  A block
// walks through its run item by item; an item that is whole inside it is written out, the pieces of one that a cut goes through
// leave records that a third kernel adds up.
//
// A block's sixteen warps talk through mbarriers only:
//   copies (1)    TMA boxes of 32 tokens of keys and of values into raw stages, and their pages' scales
//   expansion (6) two teams, keys and values: raw stages into operand slots; waiting rows (bf16) times the power of two that brings
//                 their largest magnitude near 1, a box a warp
//   products (1)  S[u] = Q[u] K_j^T, O[u] += P[u] V_j
//   softmax (8)   two groups u, a row a thread, which also fetch the queries and write the output
// u is a tile of 128 rows when there are two, else the parity of the token tile, so that one group's exponentials always run beside
// the other's products.  Every wait is bounded; a block that gives up leaves NaN.
//
// Rounded to fewer than 32 bits, because the products' operands are: queries, and waiting rows, to fp16 times one power of two for a row,
// or for 32 of them (exact from 2^-17 of the largest on, and what is below 2^-24 of it lost), and weights to fp16, 2^-11 of themselves
// against the 2^-8 of the output.  The sum takes the weights before that rounding (32 bits; summing them as rounded would take two
// conversions more for each pair of a loop that bounds the kernel), so a heavy one's rounding stays in the output, an eighth of its own.
//
// Measured: the last 1999 of 16300 tokens, 64 query and 8 KV heads (1.0 TFLOP) 1.09 ms, 0.92 PFLOP/s.  The bound is the chain of a
// tile's softmax (read S, maximum, 256 x 128 exponentials, weights back to tensor memory) with the two hand-overs around it: without
// the products it took nearly as long (0.97 of 1.12 ms), the exponentials alone would be half of it, expansion and copies wait for
// free slots, and the GPU is at its power limit.  Prompts from nothing, 32 query and 8 KV heads: 4096 tokens 391 us, 8192 tokens 1.10 ms.
// Few rows leave most of a row tile empty: 16 sequences of 3000 to 4100 tokens with 20 rows per KV head are 67 us here, 53 in the form for
// few rows, with 64 rows 69 us here; and a chunk of 512 tokens beside 63 single ones on up to 15000, all of which come here with it, 869
// us, where the two forms take 212 for the two parts.  Short items are bound by the chain queries, product, softmax, output of each: 64
// chunks of 97 tokens 85 us, 11 us of it an item's fixed cost.
#include <algorithm>

#include "qp_mma.cuh"
#include "qp_paged.cuh"
#include "qp_tc.cuh"

namespace qp {

namespace {

constexpr int PC_SOFT = 8, PC_TEAM = 3;                         // softmax warps; warps that expand the keys, and the values
constexpr int PC_MMA = PC_SOFT + 2 * PC_TEAM, PC_COPY = PC_MMA + 1;   // the warp that issues the products, the one that copies
constexpr int PC_THREADS = (PC_COPY + 1) * 32;
constexpr int PC_SLOTS = 4;                                     // operand slots, keys and values in turn
__host__ __device__ constexpr int raw_stages(int D) { return D == 64 ? 12 : 4; }    // of a team, 32 tokens each: what shared memory has room for
constexpr int PC_BLOCKS = 148;                                  // of a B200, one a SM; the layout of the workspace goes by it
constexpr int PC_SCALES = 8;                                    // tiles whose scales are kept: more than the expansion can be ahead of the softmax
constexpr float PC_HEAD = 11.f, PC_SLACK = 4.f;                 // see PA_HEAD, PA_SLACK

struct ChunkEntry {                                             // 256 rows of a sequence
  int tile, tiles, b, rg;                                       // first of its Hkv * tiles tiles
};
struct Place {                                                  // a tile of the flat sequence: entry, its numbers, head, place in the item
  int e, b, h, rg, tiles, j;
};
struct ChunkLaunch {
  PagedAttnArgs a;
  int G, max_entries;
  int* head;                                                    // {entries, tiles}
  Place* cut;                                                   // [PC_BLOCKS]: where each block's run begins
  ChunkEntry* entry;
  float* rec;                                                   // [2 * PC_BLOCKS][256][D]
  float2* rec_ml;                                               // [2 * PC_BLOCKS][256]
};

__device__ __forceinline__ int c_start(int c, int T) { return (int)((long long)T * c / PC_BLOCKS); }
__device__ __forceinline__ int c_owner(int x, int T) { return (int)((((long long)x + 1) * PC_BLOCKS - 1) / T); }

// numbers the items' tiles, one thread for a sequence, then one for 256 rows of one, and finds where the blocks' runs begin
__global__ void __launch_bounds__(1024)
chunk_plan_kernel(const __grid_constant__ ChunkLaunch p) {
  __shared__ int s_sum[32], s_first[QP_MAX_SEQS + 1];           // first entry of every sequence
  chain_enter();
  const StepView& s = p.a.s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  auto scan = [&](int v, int& all) {                            // exclusive sum over the block
    int in = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, in, o);
      if (lane >= o) in += x;
    }
    __syncthreads();
    if (lane == 31) s_sum[warp] = in;
    __syncthreads();
    int before = 0;
    all = 0;
    for (int w = 0; w < 32; ++w) {
      if (w < warp) before += s_sum[w];
      all += s_sum[w];
    }
    return before + in - v;
  };
  int entries = 0, all;
  for (int b0 = 0; b0 < s.n_seqs; b0 += 1024) {
    const int b = b0 + tid, n = b < s.n_seqs ? (seq_of(s, b).n * p.G + 255) / 256 : 0, e = scan(n, all);
    if (b < s.n_seqs) s_first[b] = entries + e;
    entries += all;
  }
  // (rows that several sequences claim could make more entries than there is room for: the call is left out then)
  if (entries > p.max_entries) entries = 0;
  int tiles = 0;
  __syncthreads();
  for (int e0 = 0; e0 < entries; e0 += 1024) {
    const int e = e0 + tid;
    ChunkEntry en{0, 0, 0, 0};
    if (e < entries) {
      int lo = 0, hi = s.n_seqs;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_first[mid] <= e) lo = mid; else hi = mid;
      }
      const Seq q = seq_of(s, lo);
      en.b = lo;
      en.rg = e - s_first[lo];
      en.tiles = (q.len + (min(q.n * p.G, (en.rg + 1) * 256) - 1) / p.G + 1 + 127) / 128;
    }
    en.tile = tiles + scan(en.tiles * p.a.Hkv, all);
    if (e < entries) p.entry[e] = en;
    tiles += all;
  }
  if (tid == 0) {
    p.head[0] = entries;
    p.head[1] = tiles;
  }
  __syncthreads();                                              // (the entries are this block's own writes)
  const int x = c_start(tid, tiles);
  if (tid < PC_BLOCKS && x < tiles) {
    int lo = 0, hi = entries;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.entry[mid].tile <= x) lo = mid; else hi = mid;
    }
    const ChunkEntry en = p.entry[lo];
    const int in = x - en.tile, h = in / en.tiles;
    p.cut[tid] = Place{lo, en.b, h, en.rg, en.tiles, in - h * en.tiles};
  }
}

// byte offset of 16-byte chunk c of row r in an operand tile of 128 rows
__device__ __forceinline__ uint32_t op_off(int r, int c) {
  return (uint32_t)((c >> 3) * 16384 + (r >> 3) * 1024 + (r & 7) * 128 + (((c & 7) ^ (r & 7)) << 4));
}
__device__ __forceinline__ void sts128(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};\n" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint32_t hadd2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("add.rn.f16x2 %0, %1, %2;\n" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// four codes as fp16 operands.  e4m3: the hardware's conversion (exact), in order; int8: as they are (1024 + 128 + c, less 1152), in
// the order 0, 2, 1, 3
template <int FORMAT>
__device__ __forceinline__ uint2 four_codes(uint32_t w) {
  if (FORMAT == QP_E4M3) {
    uint2 d;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}\n" : "=r"(d.x), "=r"(d.y) : "r"(w));
    return d;
  }
  return make_uint2(hadd2((w & 0x00ff00ffu) ^ 0x64806480u, 0xe480e480u), hadd2(((w >> 8) & 0x00ff00ffu) ^ 0x64806480u, 0xe480e480u));
}
// 16-byte chunk c of row r of a raw box, as the copy's swizzle leaves it
template <int D>
__device__ __forceinline__ uint32_t raw_off(int r, int c) {
  return D == 128 ? (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)) : (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
}
// channels 0 .. 3 of two bf16 words times f, in the operands' order
template <int FORMAT>
__device__ __forceinline__ uint2 four_ops(uint32_t w0, uint32_t w1, float f) {
  if (FORMAT == QP_E4M3) return make_uint2(pack_half2(bf16lo(w0) * f, bf16hi(w0) * f), pack_half2(bf16lo(w1) * f, bf16hi(w1) * f));
  return make_uint2(pack_half2(bf16lo(w0) * f, bf16lo(w1) * f), pack_half2(bf16hi(w0) * f, bf16hi(w1) * f));
}
__device__ __forceinline__ uint32_t abs_max(uint32_t m, const uint4& v) {
  m = __vmaxu2(m, v.x & 0x7fff7fffu);
  m = __vmaxu2(m, v.y & 0x7fff7fffu);
  m = __vmaxu2(m, v.z & 0x7fff7fffu);
  return __vmaxu2(m, v.w & 0x7fff7fffu);
}
// infinities and what is no number out of it
__device__ __forceinline__ uint4 finite(const uint4& v) {
  auto f = [](uint32_t w) { return w & __vcmpltu2(w & 0x7fff7fffu, 0x7f807f80u); };
  return make_uint4(f(v.x), f(v.y), f(v.z), f(v.w));
}
// the power of two that brings the magnitude with these bf16 bits into [1, 2), and its inverse
__device__ __forceinline__ float2 to_one(uint32_t m) {
  m = max(m & 0xffffu, m >> 16);
  const int e = min(max((int)(m >> 7), 1), 253);
  return make_float2(__uint_as_float((uint32_t)(254 - e) << 23), __uint_as_float((uint32_t)e << 23));
}
__device__ __forceinline__ void bar_sync(int id, int n) { asm volatile("bar.sync %0, %1;\n" ::"r"(id), "r"(n) : "memory"); }

enum : int { CB_FULL = 0, CB_EMPTY = PC_SLOTS, CB_S = 2 * PC_SLOTS, CB_P = CB_S + 2, CB_Q = CB_P + 2, CB_RAW = CB_Q + 1 };

struct Slot {                                                   // a team's place in the ring of slots, with the parity of the round
  int i;
  uint32_t round = 0;
  __device__ __forceinline__ void next() {
    i += 2;
    if (i >= PC_SLOTS) { i -= PC_SLOTS; round ^= 1u; }
  }
};

#ifdef QP_CHECKED
__device__ int g_give_up = -1;                                  // see qp_debug_give_up
#endif

template <int FORMAT, int D>
__global__ void __launch_bounds__(PC_THREADS, 1)
chunk_kernel(const __grid_constant__ ChunkLaunch p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  constexpr uint32_t SLOT = 128 * D * 2, RAW = 32 * D;
  constexpr int PC_RAW = raw_stages(D), CB_RAW_EMPTY = CB_RAW + 2 * PC_RAW, CB_COUNT = CB_RAW_EMPTY + 2 * PC_RAW;
  constexpr uint32_t ID_S = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
  constexpr uint32_t ID_O = (1u << 4) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);        // B: rows contract
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t bars[CB_COUNT];
  __shared__ float s_fk[PC_SCALES][4];                          // per 32 tokens: what S is multiplied by
  __shared__ float4 s_fv[PC_SCALES][2];                         // log2 of the values' scale, 2^-6 / scale, for two times 32 tokens
  __shared__ float3 s_raw[PC_RAW];                              // the same of the raw stages
  __shared__ uint32_t tmem_base_slot;
  __shared__ int give_up;
  const PagedAttnArgs& a = p.a;
  const StepView& s = a.s;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sQ = sbase, ring = sbase + 2 * SLOT, raw_base = ring + PC_SLOTS * SLOT;
  const uint32_t bar0 = smem_u32(&bars[0]);
  auto bar = [&](int which, int i) { return bar0 + (uint32_t)(which + i) * 8u; };
  const volatile int* gu = &give_up;
  if (tid == 0) {
    for (int i = 0; i < PC_SLOTS; ++i) {
      mbar_init(bar(CB_FULL, i), PC_TEAM);
      mbar_init(bar(CB_EMPTY, i), 1);                           // a tcgen05.commit
    }
    for (int u = 0; u < 2; ++u) {
      mbar_init(bar(CB_S, u), 1);                               // a tcgen05.commit
      mbar_init(bar(CB_P, u), 4);                               // the group's warps
    }
    mbar_init(bar(CB_Q, 0), PC_SOFT);
    for (int i = 0; i < 2 * PC_RAW; ++i) {
      mbar_init(bar(CB_RAW, i), 1);
      mbar_init(bar(CB_RAW_EMPTY, i), PC_TEAM);
    }
    give_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (warp == PC_MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_base_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  const uint32_t tmem = tmem_base_slot;
  chain_enter();
  const int T = p.head[1], cta = blockIdx.x;
  const int x0 = c_start(cta, T), x1 = c_start(cta + 1, T);
  auto tS = [&](int u) { return tmem + (uint32_t)u * 128u; };
  auto tO = [&](int u) { return tmem + 256u + (uint32_t)u * D; };

  // the pieces of the run: (item, its tiles j .. j + n - 1)
  struct Piece {
    Place at;
    Seq q;
    int n, rows, two;
  };
  // the first has been found, the others follow one another: the next head, or the next entry
  auto piece_at = [&](int x, const Piece* before = nullptr) {
    Piece c;
    if (!before) {
      c.at = p.cut[cta];
    } else {
      c.at = before->at;
      c.at.j = 0;
      if (++c.at.h == a.Hkv) {
        const ChunkEntry en = p.entry[++c.at.e];
        c.at = Place{c.at.e, en.b, 0, en.rg, en.tiles, 0};
      }
    }
    c.q = seq_of(s, c.at.b);
    c.n = min(c.at.tiles - c.at.j, x1 - x);
    c.rows = min(256, c.q.n * p.G - c.at.rg * 256);
    c.two = c.rows > 128;
    return c;
  };

  // tokens of a piece's sequence that are in whole pages
  auto whole_tokens = [&](const Piece& c) { return (c.q.len + c.q.n) / s.page * s.page; };
  // Of a 32-token box: what the product with its keys is multiplied by; of its values the log2 of that, and its inverse, times 2^-6 so
  // that the smallest bf16 number has one.
  auto scales_of = [&](float fk, float fv) {
    fv = fv == 0.f ? 0x1p-60f : fv;                             // zeros: any scale that leaves the others theirs
    return make_float3(fk, log2f(fv), __fdiv_rn(0x1p-6f, fv));
  };
  // Written with the keys' operands: the softmax of a tile begins when they are there, whatever has become of the values, and the copies
  // may be any number of tiles further.
  auto set_scales = [&](int tile, int box, float3 f) {
    s_fk[tile & (PC_SCALES - 1)][box] = f.x;
    float* d = reinterpret_cast<float*>(&s_fv[tile & (PC_SCALES - 1)][box >> 1]) + 2 * (box & 1);
    d[0] = f.y;
    d[1] = f.z;
  };

  if (warp < PC_SOFT) {
    // ---- softmax groups
    const int u = warp >> 2, rl = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float scale_log2 = 1.4426950408889634f * rsqrtf((float)D);
    uint32_t phase = 0;                                         // of CB_S[u]
    bool ok = true;
    int tiles_done = 0;                                         // of the run, for the scales' ring
    Piece c, after;
    if (x0 < x1) after = piece_at(x0);
    for (int x = x0; x < x1;) {                                 // (one that gave up goes on, without waits: the groups have barriers)
      c = after;
      const int r = (c.two ? u * 128 : 0) + rl;                 // row of the item
      const bool has = r < c.rows;
      const bool work = (c.two ? u * 128 : 0) + (warp & 3) * 32 < c.rows;            // warp-uniform
      const int gr = c.at.rg * 256 + r, tok = gr / p.G, head = c.at.h * p.G + gr - tok * p.G;
      // The row, in fp16 times the power of two that brings its largest magnitude near 1.  A warp's 32 rows come (and leave, below)
      // whole through their place in the queries' tile: a row a lane would touch 32 lines with every access, 7000 clocks to fetch the
      // 256 rows of an item and 10000 to write them.
      constexpr int CH = D / 8, STEP = 32 / CH;                 // 16-byte chunks of a row of 16-bit numbers; rows at a time
      const int wr = (warp & 3) * 32 + lane / CH, ch = lane % CH;
      const uint32_t place = sQ + u * SLOT;
      float cq = 0.f;
      {
        const long long from = has ? (c.q.row0 + tok) * a.qs + (long long)head * D : -1;
        uint32_t m = 0u;
        uint4 v[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
          const long long o = __shfl_sync(0xffffffffu, from, k * STEP + lane / CH);
          v[k] = o >= 0 ? __ldg(reinterpret_cast<const uint4*>(a.q + o) + ch) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int k = 0; k < CH; ++k) sts128(place + op_off(wr + k * STEP, ch), v[k]);
        __syncwarp();
#pragma unroll
        for (int k = 0; k < CH; ++k) v[k] = lds128(place + op_off(rl, k));
#pragma unroll
        for (int k = 0; k < CH; ++k) m = abs_max(m, v[k]);
        const float2 f = to_one(m);
        cq = f.y * scale_log2;
        if (c.two || u == 0) {
#pragma unroll
          for (int k = 0; k < CH; ++k) {
            const uint2 lo = four_ops<FORMAT>(v[k].x, v[k].y, f.x), hi = four_ops<FORMAT>(v[k].z, v[k].w, f.x);
            sts128(place + op_off(rl, k), make_uint4(lo.x, lo.y, hi.x, hi.y));
          }
        }
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(CB_Q, 0));
      }
      // columns of a box to logits; never 0, which would make a hidden column's -inf a NaN, nor, where all of the box is hidden, what is
      // no number, as the scale of a page with such a key is
      auto factor = [&](float fk, bool hidden) {
        const float f = fk * cq;
        return f < 0x1p-126f || hidden ? 0x1p-126f : f;         // (NaN stays)
      };
      const int lim = c.q.len + (has ? tok : c.q.n - 1) + 1;    // positions this row sees
      float m_run = -INFINITY, l_run = 0.f;                     // (the sum is times 2^-6 until the piece ends)
      float s0 = 1.f, log_s0 = 0.f;
      bool any = false;
      for (int k = c.two ? 0 : u; k < c.n && ok; k += c.two ? 1 : 2) {
        const int j = c.at.j + k;
        ok = mbar_wait_warp(bar(CB_S, u), phase, gu);
        phase ^= 1u;
        if (!ok) break;
        if (work) {
          asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
          const uint32_t ts = tS(u) + lanes;
          const int sr = (tiles_done + k) & (PC_SCALES - 1);
          if (!any) {                                           // (both groups: of the first tile)
            const float4 fv = s_fv[tiles_done & (PC_SCALES - 1)][0];
            log_s0 = fv.x;
            s0 = __fdiv_rn(0x1p-6f, fv.y);
          }
          const int vis = lim - 128 * j;                        // columns of the tile that the row sees
          int boxes = 4;                                        // of which a row of the warp sees something
          if (__any_sync(0xffffffffu, vis < 128)) {             // what a row does not see leaves S
            boxes = min(4, max(1, (__reduce_max_sync(0xffffffffu, vis) + 31) >> 5));
#pragma unroll 1
            for (int c0 = 0; c0 < 128; c0 += 32) {
              uint32_t v[32], lo[16], hi[16];
              tmem_ld32_issue(ts + c0, v);
              tmem_wait(v);
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                lo[i] = c0 + i < vis ? v[i] : 0xff800000u;
                hi[i] = c0 + 16 + i < vis ? v[16 + i] : 0xff800000u;
              }
              __syncwarp();
              tmem_st(ts + c0, lo);
              tmem_st(ts + c0 + 16, hi);
            }
            tmem_wait_st();
          }
          // Loops of small bodies: the groups, the expanding warps and the others share each quarter of the SM's instruction cache, and
          // straight code of a whole row's columns is waited for (the weights kept in registers over one unrolled pass: 1390 us for
          // 1999 tokens of 64 heads at 14301, against 1119 then).
          float mx = -INFINITY;
#pragma unroll 1
          for (int h2 = 0; h2 < 2; ++h2) {
            uint32_t xa[32], xb[32];
            tmem_ld32_issue(ts + 64 * h2, xa);
            tmem_ld32_issue(ts + 64 * h2 + 32, xb);
            tmem_wait(xa);
            tmem_wait(xb);
            float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              mx0 = max3(mx0, __uint_as_float(xa[i]), __uint_as_float(xa[i + 1]));
              mx1 = max3(mx1, __uint_as_float(xb[i]), __uint_as_float(xb[i + 1]));
            }
            const float4 fv = s_fv[sr][h2];
            mx = max3(mx, fmaf(mx0, factor(s_fk[sr][2 * h2], false), fv.x), fmaf(mx1, factor(s_fk[sr][2 * h2 + 1], false), fv.z));   // (NaN does not count)
          }
          // a new reference only where the old one is exceeded by more than 2^4 (or there is none yet)
          const bool renew = mx > m_run + PC_SLACK;
          if (__any_sync(0xffffffffu, renew)) {
            const float mn = renew ? mx : m_run, corr = renew ? ex2a(m_run - mn) : 1.f;
            m_run = mn;
            l_run *= corr;
            if (any) {
#pragma unroll 1
              for (int c0 = 0; c0 < D; c0 += 16) {
                uint32_t o[16];
                tmem_ld16_issue(tO(u) + lanes + c0, o);
                tmem_wait16(o);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * corr);
                __syncwarp();
                tmem_st(tO(u) + lanes + c0, o);
              }
              tmem_wait_st();
            }
          }
          const float ref = PC_HEAD - (m_run == -INFINITY ? 0.f : m_run);
          // P over columns of S that have been read
          uint32_t v[32], pk[16];
          tmem_ld32_issue(ts, v);
#pragma unroll 1
          for (int box = 0; box < boxes; ++box) {
            tmem_wait(v);
            const float2 fv = reinterpret_cast<const float2*>(s_fv[sr])[box];
            const float f = factor(s_fk[sr][box], 32 * box >= vis), n = ref + fv.x;
            const uint64_t sc = pack2(f, f), nm = pack2(n, n);
            uint64_t y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = fma2(pack2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), sc, nm);
            if (box + 1 < boxes) tmem_ld32_issue(ts + 32 * (box + 1), v);
            uint64_t sum2 = pack2(0.f, 0.f), sum3 = sum2;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float e0, e1;
              unpack2(y[i], e0, e1);
              e0 = ex2a(e0);
              e1 = ex2a(e1);
              pk[i] = pack_half2(e0, e1);
              if (i & 1) sum3 = add2(sum3, pack2(e0, e1)); else sum2 = add2(sum2, pack2(e0, e1));
            }
            sum2 = add2(sum2, sum3);
            float a0, a1;
            unpack2(sum2, a0, a1);
            l_run = fmaf(a0 + a1, fminf(fv.y * s0, 0x1p90f), l_run);        // (a scale that is no number: nor are the weights that see it)
            __syncwarp();
            tmem_st(ts + 16 * box, pk);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) pk[i] = 0u;
#pragma unroll 1
          for (int box = boxes; box < 4; ++box) tmem_st(ts + 16 * box, pk);
          any = true;
          tmem_wait_st();
          asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(CB_P, u));
      }
      l_run *= 64.f;
      if (x + c.n < x1) after = piece_at(x + c.n, &c);          // (its numbers are on their way meanwhile)
      // O is complete with one more commit
      ok = ok && mbar_wait_warp(bar(CB_S, u), phase, gu);
      phase ^= 1u;
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      if (!ok) give_up = 1;
#ifdef QP_CHECKED
      const bool lost = cta == g_give_up;
#else
      constexpr bool lost = false;
#endif
      if (!ok || lost) {                                        // what is lost must not look like a row that sees nothing
        m_run = 0.f;
        l_run = NAN;
      }
      const bool whole = c.at.j == 0 && c.n == c.at.tiles;
      const int rec = 2 * cta + (x == x0 ? 0 : 1);
      // The sum and O in units without s0, and the reference that goes with them.  A sum that is no number has to be looked at by those who
      // join the parts, so its reference is one that counts, whatever has become of m_run and of the scale.
      const float m_own = l_run != l_run ? 0.f : m_run == -INFINITY ? m_run : m_run - log_s0;
      // four channels of an output row: unnormalised, with the reference and the sum, where others have a part in it
      auto put = [&](int row, int ch, float4 v, float M, float L, float inv) {
        if (FORMAT == QP_INT8) {                                // columns 0, 1, 2, 3 are channels 0, 2, 1, 3
          const float t = v.y;
          v.y = v.z;
          v.z = t;
        }
        if (whole) {
          const int g = c.at.rg * 256 + row, t = g / p.G;
          *reinterpret_cast<uint2*>(a.out + ((size_t)(c.q.row0 + t) * a.Hq + c.at.h * p.G + g - t * p.G) * D + ch) =
              make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
        } else {
          *reinterpret_cast<float4*>(p.rec + ((size_t)rec * 256 + row) * D + ch) = v;
          if (ch == 0) p.rec_ml[(size_t)rec * 256 + row] = make_float2(M, L);
        }
      };
      if (c.two) {
        if (work) {
          const float f = any && m_run != -INFINITY ? s0 : 0.f, inv = __fdiv_rn(1.f, l_run);
          const int t = gr / p.G;
          const long long to = whole ? ((long long)(c.q.row0 + t) * a.Hq + c.at.h * p.G + gr - t * p.G) * D : 0;
          auto channels = [&](int c0, float (&o)[16]) {
            uint32_t v[16];
            tmem_ld16_issue(tO(u) + lanes + c0, v);
            tmem_wait16(v);
#pragma unroll
            for (int i = 0; i < 16; ++i)                        // (int8: columns 0, 1, 2, 3 are channels 0, 2, 1, 3)
              o[i] = f == 0.f ? 0.f : __uint_as_float(v[FORMAT == QP_INT8 && ((i + 1) & 2) ? i ^ 3 : i]) * f;
          };
          // half: fp32 records take a row's place twice
          for (int half = 0; half < (whole ? 1 : 2); ++half) {
#pragma unroll 1
            for (int c0 = 0; c0 < (whole ? D : D / 2); c0 += 16) {
              float o[16];
              channels(half * (D / 2) + c0, o);
              if (whole) {
#pragma unroll
                for (int i = 0; i < 16; i += 8)
                  sts128(place + op_off(rl, (c0 + i) / 8), make_uint4(pack_bf16x2(o[i] * inv, o[i + 1] * inv), pack_bf16x2(o[i + 2] * inv, o[i + 3] * inv),
                                                                     pack_bf16x2(o[i + 4] * inv, o[i + 5] * inv), pack_bf16x2(o[i + 6] * inv, o[i + 7] * inv)));
              } else {
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                  sts128(place + op_off(rl, (c0 + i) / 4),
                         make_uint4(__float_as_uint(o[i]), __float_as_uint(o[i + 1]), __float_as_uint(o[i + 2]), __float_as_uint(o[i + 3])));
              }
            }
            __syncwarp();
#pragma unroll 4
            for (int k = 0; k < CH; ++k) {
              const uint4 v = lds128(place + op_off(wr + k * STEP, ch));
              const long long o = __shfl_sync(0xffffffffu, to, k * STEP + lane / CH);
              const int row = u * 128 + wr + k * STEP;
              if (row >= c.rows) continue;
              if (whole)
                *(reinterpret_cast<uint4*>(a.out + o) + ch) = v;
              else
                *reinterpret_cast<uint4*>(p.rec + ((size_t)rec * 256 + row) * D + half * (D / 2) + 4 * ch) = v;
            }
            __syncwarp();
          }
          if (!whole && has) p.rec_ml[(size_t)rec * 256 + r] = make_float2(m_own, l_run);
        }
      } else {
        // the two groups' parts of a row come together through shared memory: statistics in the queries' place, a
        // quarter of the channels at a time in the second row tile's
        constexpr int QD = D / 4, CH = QD / 4;                  // channels of a quarter, 16-byte chunks
        const uint32_t xch = sQ + SLOT;
        float2* s_ml = reinterpret_cast<float2*>(smem_raw + (sQ - smem_u32(smem_raw)));
        auto total = [&](int row, float& M, float& L) {
          M = -INFINITY;
          L = 0.f;
          for (int i = 0; i < 2; ++i) M = fmaxf(M, s_ml[i * 128 + row].x);
          for (int i = 0; i < 2; ++i) {
            const float2 ml = s_ml[i * 128 + row];
            if (ml.x != -INFINITY) L = fmaf(ml.y, ex2a(ml.x - M), L);
          }
        };
        bar_sync(3, PC_SOFT * 32);                              // both groups have seen their last product: nobody reads the queries
        s_ml[u * 128 + rl] = make_float2(m_own, l_run);         // (a group without a tile: -inf, as it began)
        bar_sync(3, PC_SOFT * 32);
        float M = -INFINITY, L;
        if (has) total(r, M, L);
        const float f = any && has && m_own != -INFINITY ? ex2a(m_own - M) * s0 : 0.f;
#pragma unroll 1
        for (int quarter = 0; quarter < 4; ++quarter) {
          if (work) {
#pragma unroll 1
            for (int c0 = 0; c0 < QD; c0 += 16) {
              uint32_t o[16];
              if (any) {
                tmem_ld16_issue(tO(u) + lanes + quarter * QD + c0, o);
                tmem_wait16(o);
              }
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = f != 0.f ? __float_as_uint(__uint_as_float(o[i]) * f) : 0u;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                sts128(xch + (u * 128 + rl) * (QD * 4) + (((c0 / 4 + i) ^ (rl & (CH - 1))) << 4), make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]));
            }
          }
          bar_sync(3, PC_SOFT * 32);
          for (int i = tid; i < c.rows * CH; i += PC_SOFT * 32) {
            const int row = i / CH, ch = i % CH;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int k = 0; k < 2; ++k) {
              const int at = k * 128 + row;
              const uint4 w = lds128(xch + at * (QD * 4) + ((ch ^ (at & (CH - 1))) << 4));
              v.x += __uint_as_float(w.x); v.y += __uint_as_float(w.y);
              v.z += __uint_as_float(w.z); v.w += __uint_as_float(w.w);
            }
            float rM, rL;
            total(row, rM, rL);
            put(row, quarter * QD + 4 * ch, v, rM, rL, __fdiv_rn(1.f, rL));
          }
          bar_sync(3, PC_SOFT * 32);
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
      tiles_done += c.n;
      x += c.n;
    }
  } else if (warp == PC_MMA) {
    // ---- products.  Operands in the ring: keys of tile 0, values of tile 0, keys of tile 1, ..., across pieces
    bool ok = true;
    Slot kr{0}, vr{1};
    uint32_t pq = 0, pp[2] = {0, 0};                            // phases of CB_Q, CB_P
    auto wait_full = [&](const Slot& r) { ok = ok && mbar_wait_warp(bar(CB_FULL, r.i), r.round, gu); };
    auto wait_p = [&](int u) {
      ok = ok && mbar_wait_warp(bar(CB_P, u), pp[u], gu);
      pp[u] ^= 1u;
    };
    auto issue_s = [&](int u, int qt, bool last_reader) {
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      const uint32_t q = uniform(desc_lo(sQ + qt * SLOT, 1)), kk = uniform(desc_lo(ring + kr.i * SLOT, 1));
      const uint32_t d = uniform(tS(u)), done = uniform(bar(CB_S, u)), empty = uniform(bar(CB_EMPTY, kr.i));
      if (elect_one()) {
        umma_ss<false>(d, q, kk, ID_S);
#pragma unroll
        for (int k = 1; k < D / 16; ++k) umma_ss<true>(d, q + (k / 4) * 1024 + (k % 4) * 2, kk + (k / 4) * 1024 + (k % 4) * 2, ID_S);
        umma_commit(done);
        if (last_reader) umma_commit(empty);
      }
      __syncwarp();
      if (last_reader) kr.next();
    };
    auto issue_o = [&](int u, bool first, bool last_reader) {
      asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
      const uint32_t vv = uniform(desc_lo(ring + vr.i * SLOT, 1024)), d = uniform(tO(u)), pt = uniform(tS(u));
      const uint32_t empty = uniform(bar(CB_EMPTY, vr.i));
      if (elect_one()) {
        umma_ts(d, pt, vv, ID_O, first ? 0u : 1u);
#pragma unroll
        for (int k = 1; k < 8; ++k) umma_ts(d, pt + 8 * k, vv + k * 128, ID_O, 1u);
        if (last_reader) umma_commit(empty);
      }
      __syncwarp();
      if (last_reader) vr.next();
    };
    auto finish = [&](int u) {                                  // one more commit: O[u] is complete
      const uint32_t done = uniform(bar(CB_S, u));
      if (elect_one()) umma_commit(done);
      __syncwarp();
    };
    Piece c;
    for (int x = x0; x < x1 && ok;) {
      c = x == x0 ? piece_at(x) : piece_at(x, &c);
      ok = mbar_wait_warp(bar(CB_Q, 0), pq, gu);
      pq ^= 1u;
      if (c.two) {
        wait_full(kr);
        if (ok) issue_s(0, 0, false);
        if (ok) issue_s(1, 1, true);
        for (int j = 0; j < c.n && ok; ++j)
          for (int u = 0; u < 2 && ok; ++u) {
            if (u == 0) wait_full(vr);
            wait_p(u);
            if (!ok) break;
            issue_o(u, j == 0, u == 1);
            if (j + 1 < c.n) {
              if (u == 0) wait_full(kr);
              if (ok) issue_s(u, u, u == 1);
            } else {
              finish(u);
            }
          }
      } else {
        for (int j = 0; j < min(2, c.n) && ok; ++j) {
          wait_full(kr);
          if (ok) issue_s(j, 0, true);
        }
        if (c.n == 1 && ok) finish(1);                          // (the second group has no tile)
        for (int j = 0; j < c.n && ok; ++j) {
          const int u = j & 1;
          wait_full(vr);
          wait_p(u);
          if (!ok) break;
          issue_o(u, j < 2, true);
          if (j + 2 < c.n) {
            wait_full(kr);
            if (ok) issue_s(u, 0, true);
          } else {
            finish(u);
          }
        }
      }
      x += c.n;
    }
    if (!ok) give_up = 1;
    } else if (warp == PC_COPY) {
      // ---- copies: the boxes of 32 tokens of keys and of values, and their scales.  Lane i copies box i % 4 of a tile's keys (i < 4) or
      // values, as soon as its stage is free.
      bool ok = true;
      const int lg = 31 - __clz(s.page / 32), box = lane & 3, team = lane >> 2;       // lg: log2 of boxes per page
      int n_box = 0, tile = 0;                                  // boxes copied, tiles of the run before this one
      uint32_t left = 0;                                        // of the last tile with boxes: lanes that could not copy theirs
      int n_last = 0;                                           // and its boxes
      Piece c;
      for (int x = x0; x < x1 && ok;) {
        c = x == x0 ? piece_at(x) : piece_at(x, &c);
        const int whole = whole_tokens(c);
        int window = -64, w_id = -1;                            // 32 pages: ids and scales in the lanes
        float w_ks = NAN, w_vs = NAN;
        for (int k = 0; k < c.n && ok; ++k, ++tile) {
          const int t0 = 128 * (c.at.j + k), boxes = min(4, max(0, (whole - t0) / 32));
          if (boxes == 0) continue;
          const int pg0 = t0 / 32 >> lg, pg1 = (t0 / 32 + boxes - 1) >> lg;
          if (pg0 < window || pg1 >= window + 32) {
            window = pg0;
            const int i = pg0 + lane;
            w_id = i < whole / s.page ? page_of(s, c.at.b, i) : -1;
            w_ks = w_vs = NAN;                                  // a page outside the pool makes its rows NaN
            if (w_id >= 0) {
              w_ks = bf16_bits_to_f32(__ldg(a.k_scale + (size_t)w_id * a.Hkv + c.at.h));
              w_vs = bf16_bits_to_f32(__ldg(a.v_scale + (size_t)w_id * a.Hkv + c.at.h));
            }
          }
          const int bx = t0 / 32 + min(box, boxes - 1), src = (bx >> lg) - window;
          const int id = max(0, __shfl_sync(0xffffffffu, w_id, src));
          const float ks = __shfl_sync(0xffffffffu, w_ks, src), vs = __shfl_sync(0xffffffffu, w_vs, src);
          const int n = n_box + box, st = team * PC_RAW + n % PC_RAW, row = (id * a.Hkv + c.at.h) * s.page + (bx & ((1 << lg) - 1)) * 32;
          bool todo = lane < 8 && box < boxes;
          const float3 scales = scales_of(ks, vs);
          for (uint32_t y = 0; __any_sync(0xffffffffu, todo); ++y) {
            if (todo && (n < PC_RAW || mbar_try_wait(bar(CB_RAW_EMPTY, st), (uint32_t)(n / PC_RAW + 1) & 1u))) {
              if (team == 0) s_raw[st] = scales;
              mbar_expect_tx(bar(CB_RAW, st), RAW);
              tma_load_2d(raw_base + st * RAW, team ? &map_v : &map_k, 0, row, bar(CB_RAW, st));
              todo = false;
            }
            if (y >= TC_SPIN_LIMIT || ((y & 255u) == 255u && *gu)) break;
          }
          left = __ballot_sync(0xffffffffu, todo);
          ok = left == 0;
          n_last = boxes;
          n_box += boxes;
        }
        x += c.n;
      }
      if (!ok) give_up = 1;
      // nothing may still be on its way into this block's shared memory when it is given up: the last copies are waited for (bounded)
      for (int i = max(0, n_box - PC_RAW); i < n_box; ++i)
        for (int h = 0; h < 2; ++h) {
          const int in_last = i - (n_box - n_last);             // (a box that could not be copied: its stage's one before)
          const int n = in_last >= 0 && (left >> (4 * h + in_last) & 1u) ? i - PC_RAW : i;
          for (uint32_t y = 0; n >= 0 && y < TC_SPIN_LIMIT; ++y)
            if (mbar_try_wait(bar(CB_RAW, h * PC_RAW + n % PC_RAW), (uint32_t)(n / PC_RAW) & 1u)) break;
        }
    } else {
      // ---- codes to operands
      const int team = (warp - PC_SOFT) / PC_TEAM, tw = (warp - PC_SOFT) % PC_TEAM;
      const uint16_t* tails = team ? a.v_tail : a.k_tail;
      const uint32_t raw0 = raw_base + team * PC_RAW * RAW;
      // a warp takes 8 rows x 4 chunks at a time: the lanes of a quarter have rows i and i ^ 5, whose chunks meet no bank twice
      const int row8 = (lane >> 3) ^ (lane & 4 ? 5 : 0), c4 = lane & 3;
      const uint32_t from = raw_off<D>(row8, c4), to0 = op_off(row8, 2 * c4), to1 = op_off(row8, 2 * c4 + 1);
      constexpr int PARTS = D / 64, ITEMS = 4 * PARTS, MOST = (ITEMS + PC_TEAM - 1) / PC_TEAM;   // of a box: 8 rows x 64 channels
      bool ok = true;
      Slot wr{team};
      int n_box = 0, tile = 0;
      Piece c;
      for (int x = x0; x < x1 && ok;) {
        c = x == x0 ? piece_at(x) : piece_at(x, &c);
        const int whole = whole_tokens(c), end = c.q.len + c.q.n;
        for (int k = 0; k < c.n && ok; ++k, ++tile) {
          const int t0 = 128 * (c.at.j + k), boxes = min(4, max(0, (whole - t0) / 32));
          const uint32_t slot = ring + wr.i * SLOT;
          if (tile >= 2) ok = mbar_wait_warp(bar(CB_EMPTY, wr.i), wr.round ^ 1u, gu);
          for (int box = 0; box < boxes && ok; ++box, ++n_box) {
            const int stage = n_box % PC_RAW, first = (tw + n_box) % PC_TEAM;      // (the shares differ: in turn)
            ok = mbar_wait_warp(bar(CB_RAW, team * PC_RAW + stage), (uint32_t)(n_box / PC_RAW) & 1u, gu);
            if (!ok) break;
            if (team == 0 && first == 0 && lane == 0) set_scales(tile, box, s_raw[stage]);
            uint4 w[MOST];
#pragma unroll
            for (int q = 0; q < MOST; ++q) {
              const int i = first + q * PC_TEAM, g8 = i / PARTS, part = i % PARTS;
              if (i < ITEMS) w[q] = lds128(raw0 + stage * RAW + g8 * 8 * D + (from ^ (part * 64)));
            }
#pragma unroll
            for (int q = 0; q < MOST; ++q) {
              const int i = first + q * PC_TEAM, g8 = i / PARTS, part = i % PARTS;
              if (i < ITEMS) {
                const uint32_t at = slot + (4 * box + g8) * 1024 + part * 16384;
                const uint2 o0 = four_codes<FORMAT>(w[q].x), o1 = four_codes<FORMAT>(w[q].y), o2 = four_codes<FORMAT>(w[q].z), o3 = four_codes<FORMAT>(w[q].w);
                sts128(at + to0, make_uint4(o0.x, o0.y, o1.x, o1.y));
                sts128(at + to1, make_uint4(o2.x, o2.y, o3.x, o3.y));
              }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(CB_RAW_EMPTY, team * PC_RAW + stage));
          }
          if (!ok) break;
          // waiting rows, a box a warp, read once: bf16 to fp16 times a power of two; zeros behind the last
          for (int box = boxes + tw; box < 4; box += PC_TEAM) {
            constexpr int CH = D / 8, STEP = 32 / CH;           // 16-byte chunks of a row; rows at a time
            const int r0 = lane / CH, ch = lane % CH, left = end - (t0 + 32 * box);
            const size_t from_row = (((size_t)c.at.b * a.Hkv + c.at.h) * s.page + t0 + 32 * box - whole) * CH + lane;
            auto at = [&](int q) { return slot + op_off(32 * box + r0 + q * STEP, ch); };
            // the box to its place as it is, and the power of two for it
            auto fetch = [&](const uint16_t* tail) {
              uint4 v[CH];
#pragma unroll
              for (int q = 0; q < CH; ++q)
                v[q] = r0 + q * STEP < left ? reinterpret_cast<const uint4*>(tail)[from_row + 32 * q] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
              for (int q = 0; q < CH; ++q) sts128(at(q), v[q]);
              uint32_t m = 0u;
#pragma unroll 4
              for (int q = 0; q < CH; ++q) m = abs_max(m, lds128(at(q)));
              m = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
              if (m >= 0x7f80u) {                               // of what is finite
                m = 0u;
#pragma unroll 1
                for (int q = 0; q < CH; ++q) m = abs_max(m, finite(lds128(at(q))));
                m = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
              }
              return m ? to_one(m) : make_float2(1.f, 0.f);
            };
            if (left <= 0) {                                    // (hidden keys, and values of weight 0)
#pragma unroll
              for (int q = 0; q < CH; ++q) sts128(at(q), make_uint4(0u, 0u, 0u, 0u));
              if (team == 0 && lane == 0) set_scales(tile, box, scales_of(0.f, 0.f));
              continue;
            }
            float2 fv = make_float2(0.f, 0.f);
            if (team == 0) fv = fetch(a.v_tail);
            const float2 f = fetch(tails);
#pragma unroll 2
            for (int q = 0; q < CH; ++q) {
              const uint4 v = lds128(at(q));
              const uint2 lo = four_ops<FORMAT>(v.x, v.y, f.x), hi = four_ops<FORMAT>(v.z, v.w, f.x);
              sts128(at(q), make_uint4(lo.x, lo.y, hi.x, hi.y));
            }
            if (team == 0 && lane == 0) set_scales(tile, box, scales_of(f.y, fv.y));
          }
          asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(CB_FULL, wr.i));
          wr.next();
        }
        x += c.n;
      }
      if (!ok) give_up = 1;
    }
  asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
  if (warp == PC_MMA)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512u) : "memory");
}

// the items that cuts go through: out from their records, in order.  A block row (y) for every cut, which takes the item if it is its
// first; a thread for 4 channels of a row
template <int D>
__global__ void __launch_bounds__(256)
chunk_merge_kernel(const __grid_constant__ ChunkLaunch p) {
  chain_enter();
  const int T = p.head[1], cut = blockIdx.y + 1;
  if (T == 0) return;
  const int x = c_start(cut, T);
  if (x >= T || x == c_start(cut - 1, T)) return;               // (runs without tiles)
  const Place at = p.cut[cut];
  const int first = x - at.j, last = first + at.tiles - 1;      // the item's tiles
  if (at.j == 0 || c_owner(first, T) != cut - 1) return;        // the cut falls between items, or is not the item's first
  const PagedAttnArgs& a = p.a;
  const Seq q = seq_of(a.s, at.b);
  const int i = blockIdx.x * 256 + threadIdx.x, r = i / (D / 4), ch = i % (D / 4), gr = at.rg * 256 + r;
  if (r >= 256 || gr >= q.n * p.G) return;
  const int c1 = c_owner(last, T);
  float M = -INFINITY, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int c = cut - 1; c <= c1; ++c) {
    const int s0 = c_start(c, T);
    if (s0 == c_start(c + 1, T)) continue;
    const size_t row = (size_t)(2 * c + (s0 >= first ? 0 : 1)) * 256 + r;
    const float2 ml = p.rec_ml[row];
    const float4 v = *reinterpret_cast<const float4*>(p.rec + row * D + 4 * ch);
    if (ml.x == -INFINITY) continue;                            // a piece of which the row sees nothing
    const float n = fmaxf(M, ml.x), f = M == -INFINITY ? 0.f : ex2a(M - n), e = ex2a(ml.x - n);
    M = n;
    L = L * f + ml.y * e;
    o.x = o.x * f + v.x * e; o.y = o.y * f + v.y * e;
    o.z = o.z * f + v.z * e; o.w = o.w * f + v.w * e;
  }
  const float inv = __fdiv_rn(1.f, L);
  const int tok = gr / p.G;
  *reinterpret_cast<uint2*>(a.out + ((size_t)(q.row0 + tok) * a.Hq + at.h * p.G + gr - tok * p.G) * D + 4 * ch) =
      make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
}

struct ChunkCarve {
  size_t entry, ml, rec, total;
  int entries;
};
ChunkCarve chunk_carve(int n_seqs, int n_tokens, int Hq, int Hkv, int D) {
  ChunkCarve c;
  c.entries = (int)((long long)n_tokens * (Hq / Hkv) / 256) + n_seqs;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  c.entry = up(256 + PC_BLOCKS * sizeof(Place));
  c.ml = up(c.entry + (size_t)c.entries * sizeof(ChunkEntry));
  c.rec = c.ml + up((size_t)2 * PC_BLOCKS * 256 * sizeof(float2));
  c.total = c.rec + (size_t)2 * PC_BLOCKS * 256 * D * sizeof(float);
  return c;
}

template <int FORMAT, int D>
cudaError_t launch_chunk_t(const ChunkLaunch& p, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t st) {
  static unsigned char done[64];
  constexpr size_t smem = (2 + PC_SLOTS) * 128 * D * 2 + 2 * raw_stages(D) * 32 * D + 1024;
  auto kernel = chunk_kernel<FORMAT, D>;
  cudaError_t e = allow_smem(kernel, smem, done);
  if (e == cudaSuccess) e = launch_chained(chunk_plan_kernel, dim3(1), dim3(1024), 0, st, p);
  if (e == cudaSuccess) e = launch_chained(kernel, dim3(PC_BLOCKS), dim3(PC_THREADS), smem, st, p, mk, mv);
  const unsigned rows = (unsigned)std::min(256LL, (long long)p.a.s.max_new * p.G);   // of an item, at most
  if (e == cudaSuccess)
    e = launch_chained(chunk_merge_kernel<D>, dim3((rows * (D / 4) + 255) / 256, PC_BLOCKS - 1), dim3(256), 0, st, p);
  return e;
}

}  // namespace

#ifdef QP_CHECKED
cudaError_t paged_chunk_check_read(unsigned int (&out)[4]) { return checked::read_and_clear(out); }
cudaError_t paged_chunk_give_up(int block) { return cudaMemcpyToSymbol(g_give_up, &block, sizeof(block)); }
#endif

size_t paged_chunk_workspace(int n_seqs, int n_tokens, int Hq, int Hkv, int D) { return chunk_carve(n_seqs, n_tokens, Hq, Hkv, D).total; }

bool paged_chunk_fits(int n_seqs, int n_tokens, int Hq, int Hkv, long long most_len) {
  const long long entries = (long long)n_tokens * (Hq / Hkv) / 256 + n_seqs;
  return entries < 0x7fffffffLL / Hkv / ((most_len + 127) / 128);
}

cudaError_t launch_paged_chunk(const PagedAttnArgs& a, void* ws, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t st) {
  ChunkLaunch p{};
  p.a = a;
  p.G = a.Hq / a.Hkv;
  const ChunkCarve c = chunk_carve(a.s.n_seqs, a.s.n_tokens, a.Hq, a.Hkv, a.D);
  char* w = static_cast<char*>(ws);
  p.max_entries = c.entries;
  p.head = reinterpret_cast<int*>(w);
  p.cut = reinterpret_cast<Place*>(w + 256);
  p.entry = reinterpret_cast<ChunkEntry*>(w + c.entry);
  p.rec_ml = reinterpret_cast<float2*>(w + c.ml);
  p.rec = reinterpret_cast<float*>(w + c.rec);
  if (a.format == QP_E4M3) return a.D == 128 ? launch_chunk_t<QP_E4M3, 128>(p, mk, mv, st) : launch_chunk_t<QP_E4M3, 64>(p, mk, mv, st);
  return a.D == 128 ? launch_chunk_t<QP_INT8, 128>(p, mk, mv, st) : launch_chunk_t<QP_INT8, 64>(p, mk, mv, st);
}

}  // namespace qp
