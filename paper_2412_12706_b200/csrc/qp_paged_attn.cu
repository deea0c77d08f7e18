// Attention of a step's new tokens over a paged cache in 8 bits (qp_paged_attn): a few rows per KV head.
//
// With one new token a sequence the cache's bytes are the floor: 2 D bytes a token and KV head against 4 G D flop.  The products run on
// mma.sync (m16n8k16, fp16): tokens, then channels, are the 16 rows, the G n query rows of a KV head the 8 columns, so a code is turned
// into an fp16 operand once whatever G is.
//   e4m3   the hardware's conversion, two codes at a time
//   int8   the code xor 128 in a lane of 16 bits is the subnormal fp16 number (c + 128) 2^-24; the 128 come off again through the
//          sum of the query (keys) and of the weights (values)
// so a pair of operands costs one to two instructions and no multiplication; the page's scales meet 32-bit accumulators.
//
// Work: every (sequence, KV head, 8 NB query rows) is an item of ceil(tokens of whole pages / 32) tiles followed by one for every 16
// waiting rows.  The tiles of all items are one sequence, cut into one equal run for each warp of the grid, found by each block from
// the lengths on the device (the host does not know them, so a captured call serves every later step).  A warp shares nothing: it
// copies its tiles by TMA into its own ring (two boxes of 32 tokens, swizzled so that the reads below meet no bank twice) and leaves
// one record (maximum, sum, O) for the pages and one for the waiting rows of every item it touches; a second kernel adds them up.
// (Neighbouring runs in one block, whose warps join their records in shared memory first: the merge of 16 sequences with 20 rows per KV
// head 7.5 -> 6.1 us, the kernel before it 46 -> 48, and one sequence of 2000 tokens 8.2 -> 11.4 in all.  So records are a warp's.)
//
// Waiting rows are bf16 and are multiplied as such, the weights as the sum of two bf16 numbers.
//
// Rounded to fewer than 32 bits, because the products' operands are: queries, to fp16 times one power of two for a row (exact from 2^-17
// of the row's largest on, and what is below 2^-24 of it lost), and the weights of pages, to fp16, 2^-11 of themselves against the 2^-8 of
// the output.  The sum takes the weights as rounded, so a heavy one's rounding cancels.
//
// Measured over changing inputs: 64 sequences of up to 16000 tokens (1.1 GB) 194 us, 5.6 TB/s, bound by HBM; 8 sequences of 32000 in
// int8 (511 MB) 97 us, 5.3 TB/s; one of 2000 tokens 10.2 us (8.2 of one cache in L2), two launches and three dependent reads (lengths,
// page, tile).  More rows per KV head are bound by the chain of dependent instructions of a tile (conversion, product, softmax, product)
// in the two warps that a scheduler has, 255 registers each: 16 sequences of 3000 to 4100 tokens, 8 / 16 / 20 / 24 / 32 rows 38 / 44 /
// 53 / 53 / 57 us against 18 for the bytes, issue slots 36 %, tensor pipe 28 % (at 20).
#include <algorithm>

#include "qp_mma.cuh"
#include "qp_paged.cuh"
#include "qp_tc.cuh"

namespace qp {

namespace {

// BUSY: calls with 64 (sequence, KV head) pairs and more.  Warps of a block and copy stages of a warp, and registers of a thread:
//   8 rows    busy: twelve warps, which hide more of a tile's chain of dependent steps (64 sequences of up to 16000 tokens: 201 -> 188
//             us, D = 64 125 -> 107; 64 of 1000: 36.7 -> 35.3), but fill the SM's registers, so that neither the merge nor the next
//             call's blocks come in beside them (one sequence of 2000 tokens: 8.2 us against 10.7)
//   16 rows   else 208 registers, which leave room for a block of the merge (one sequence of 3000 to 4100 tokens with 4 drafts 13.4 us,
//             against 15.4), busy 255 (16 of them with 8 drafts 52.5 us, against 55.7); D = 64 needs 202, so there is one form of it
//   24 rows   255, where D = 128 spills three to nine of them: with 208 it spills far more (16 sequences with 5 drafts 50 -> 58 us)
__host__ __device__ constexpr int pa_warps(int nb, int busy) { return nb == 1 && busy ? 12 : 8; }
__host__ __device__ constexpr int pa_stages(int nb, int busy) { return nb == 1 && busy ? 2 : 3; }
__host__ __device__ constexpr int pa_registers(int nb, int busy) { return nb == 1 && busy ? 168 : nb < 3 && !busy ? 208 : 255; }
constexpr int PA_MAX_SEQS = 2048;
constexpr int PA_SMS = 148;                                     // of a B200; the layout of the workspace goes by it
constexpr int PA_WORKERS = PA_SMS * pa_warps(1, 1);            // most of a launch
constexpr float PA_HEAD = 11.f;                                 // weights are held against the reference times 2^-11, to use fp16's upper range
constexpr float PA_SLACK = 4.f;                                 // a maximum is renewed when it is exceeded by 2^4

// what the kernels of a call share, computed on the device: for each sequence its first tile and its first item
struct SeqBase {
  int tile, item;
};
struct PagedLaunch {
  PagedAttnArgs a;
  int G, RB;                    // query heads per KV head, rows of an item
  int n_workers, min_tiles;
  int max_items;                // that the workspace has records for
  float* rec;                   // [slot][RB][D]
  float2* rec_ml;               // [slot][RB]
  SeqBase* base;                // [n_seqs + 1]
};

// tiles of one item of a sequence, and items per KV head
struct Shape {
  int page_tiles, tail_tiles, row_blocks;
};
__device__ __forceinline__ Shape shape_of(const Seq& q, int page, int G, int RB) {
  Shape s{0, 0, 0};
  if (q.n > 0) {
    const int end = q.len + q.n, whole = end / page * page;
    s.page_tiles = whole / 32;
    s.tail_tiles = (end - whole + 15) / 16;
    s.row_blocks = (q.n * G + RB - 1) / RB;
  }
  return s;
}
// the run of worker w: [w T / W, (w + 1) T / W); the worker that has tile x
__device__ __forceinline__ int run_start(int w, int T, int W) { return (int)((long long)w * T / W); }
__device__ __forceinline__ int owner_of(int x, int T, int W) {
  if (T < 1 << 20) return (int)(((uint32_t)(x + 1) * (uint32_t)W - 1u) / (uint32_t)T);       // W <= 2^11: a short division will do
  return (int)((((long long)x + 1) * W - 1) / T);
}
__device__ __forceinline__ int workers_of(const PagedLaunch& p, int T) {
  return max(1, min(p.n_workers, (T + p.min_tiles - 1) / p.min_tiles));
}

__device__ __forceinline__ uint32_t movmatrix(uint32_t v) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(d) : "r"(v));
  return d;
}
// fp16 operands of the four codes of w, see above: of two pairs of keys' channels (x: the b0 of a product, y: its b1), and of two
// tokens' values of a channel (x) and of the next (y)
__device__ __forceinline__ uint2 int8_codes(uint32_t w) { return make_uint2((w & 0x00ff00ffu) ^ 0x00800080u, ((w >> 8) & 0x00ff00ffu) ^ 0x00800080u); }
__device__ __forceinline__ uint2 e4m3_codes(uint32_t w) {
  uint2 d;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}\n" : "=r"(d.x), "=r"(d.y) : "r"(w));
  return d;
}
template <int FORMAT>
__device__ __forceinline__ uint2 key_codes(uint32_t w) { return FORMAT == QP_E4M3 ? e4m3_codes(w) : int8_codes(w); }
template <int FORMAT>
__device__ __forceinline__ uint2 value_codes(uint32_t w) { return FORMAT == QP_E4M3 ? e4m3_codes(__byte_perm(w, 0u, 0x3120)) : int8_codes(w); }
template <int FORMAT>
constexpr float kCodeUnit = FORMAT == QP_E4M3 ? 1.f : 0x1p24f;

// The swizzles of the copies: 16-byte chunk c of row r of a tile whose rows are 64 or 128 bytes
template <int ROW>
__device__ __forceinline__ uint32_t swz(int r, int c) {
  return ROW == 128 ? (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)) : (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
}
// the token of a group of 8 that row i of a product's operand stands for.  Rows of 128 bytes: neighbouring rows are four tokens apart,
// so that the eight lanes that read at a time find eight different chunks.
template <int D>
__device__ __forceinline__ int token_of(int i) { return D == 128 ? (i & 1) * 4 + (i >> 1) : i; }

#ifdef QP_CHECKED
__device__ int g_give_up = -1;                                  // see qp_debug_give_up
#endif

template <int FORMAT, int D, int NB, int BUSY>
__global__ void __maxnreg__(pa_registers(NB, BUSY))
paged_decode_kernel(const __grid_constant__ PagedLaunch p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                    const __grid_constant__ CUtensorMap map_kt, const __grid_constant__ CUtensorMap map_vt) {
  constexpr int RB = 8 * NB, KS = D / 16, PA_WARPS = pa_warps(NB, BUSY), PA_STAGES = pa_stages(NB, BUSY), PA_THREADS = PA_WARPS * 32;
  constexpr uint32_t SLOT = 64 * D, HALF_SLOT = SLOT / 2;       // keys, then values: 32 tokens of codes, or 16 of bf16
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t bars[PA_WARPS * PA_STAGES];
  __shared__ float2 s_scale[PA_WARPS * PA_STAGES];
  __shared__ SeqBase s_base[PA_MAX_SEQS + 1];
  __shared__ int s_sum[2][PA_WARPS];
  __shared__ int give_up;
  const PagedAttnArgs& a = p.a;
  const StepView& s = a.s;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), g = lane >> 2, t = lane & 3;
  const uint32_t ring = ((smem_u32(smem_raw) + 1023u) & ~1023u) + (uint32_t)warp * PA_STAGES * SLOT;
  const uint32_t bar0 = smem_u32(&bars[warp * PA_STAGES]);
  if (lane == 0)
    for (int i = 0; i < PA_STAGES; ++i) mbar_init(bar0 + 8 * i, 1);
  if (tid == 0) give_up = 0;
  asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  chain_enter();

  // ---- first tile and first item of every sequence
  {
    int tiles = 0, items = 0;                                   // of the sequences before this round's
    for (int b0 = 0; b0 < s.n_seqs; b0 += PA_THREADS) {
      const int b = b0 + tid;
      int nt = 0, ni = 0;
      if (b < s.n_seqs) {
        const Shape sh = shape_of(seq_of(s, b), s.page, p.G, RB);
        ni = a.Hkv * sh.row_blocks;
        nt = ni * (sh.page_tiles + sh.tail_tiles);
      }
      int ct = nt, ci = ni;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, ct, o), y = __shfl_up_sync(0xffffffffu, ci, o);
        if (lane >= o) { ct += x; ci += y; }
      }
      if (lane == 31) { s_sum[0][warp] = ct; s_sum[1][warp] = ci; }
      __syncthreads();
      int bt = tiles, bi = items;
      for (int w = 0; w < PA_WARPS; ++w) {
        if (w < warp) { bt += s_sum[0][w]; bi += s_sum[1][w]; }
        tiles += s_sum[0][w];
        items += s_sum[1][w];
      }
      if (b < s.n_seqs) s_base[b] = SeqBase{bt + ct - nt, bi + ci - ni};
      __syncthreads();
    }
    // (rows that several sequences claim could ask for more records than there are: the call is left out then)
    if (tid == 0) s_base[s.n_seqs] = SeqBase{items <= p.max_items ? tiles : 0, items};
    __syncthreads();
    if (blockIdx.x == 0)
      for (int b = tid; b <= s.n_seqs; b += PA_THREADS) p.base[b] = s_base[b];
  }
  const int T = s_base[s.n_seqs].tile, W = workers_of(p, T);
  const int worker = warp * gridDim.x + blockIdx.x;             // (neighbouring runs on different SMs)
  if (T == 0 || worker >= W) return;
  const int x0 = run_start(worker, T, W), x1 = run_start(worker + 1, T, W);
  // sequence of tile x
  auto seq_at = [&](int x) {
    int lo = 0, hi = s.n_seqs;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_base[mid].tile <= x) lo = mid; else hi = mid;
    }
    return lo;
  };

  // ---- the copies run PA_STAGES tiles ahead of the products, across items and sequences
  struct Cursor {
    int x, b, h, j;                                             // next tile; its sequence, head and place in its item
    int page_tiles, tiles, row_blocks, rb;
    int end;                                                    // tile at which the sequence ends
    int first_page, page_lane;                                  // the 32 pages whose ids the lanes hold
    float ks_lane, vs_lane;
    bool fresh = false;
  } c;
  auto enter = [&](int x) {                                     // the cursor to tile x
    c.b = seq_at(x);
    const Shape sh = shape_of(seq_of(s, c.b), s.page, p.G, RB);
    c.page_tiles = sh.page_tiles;
    c.tiles = sh.page_tiles + sh.tail_tiles;
    c.row_blocks = sh.row_blocks;
    const int in = x - s_base[c.b].tile, item = in / c.tiles;
    c.j = in - item * c.tiles;
    c.h = item / c.row_blocks;
    c.rb = item - c.h * c.row_blocks;
    c.end = s_base[c.b + 1].tile;
    c.first_page = -64;
  };
  const int lg_tp = 31 - __clz(s.page / 32);                    // log2 of tiles per page
  auto issue = [&](int k) {                                     // the k-th tile of the run
    const int slot = k % PA_STAGES;
    const uint32_t bar = bar0 + 8 * slot, dst = ring + slot * SLOT;
    if (c.j < c.page_tiles) {
      const int pg = c.j >> lg_tp;
      if ((unsigned)(pg - c.first_page) >= 32u) {               // the next 32 pages of this head
        c.first_page = pg;
        const int i = pg + lane;
        c.page_lane = i < c.page_tiles >> lg_tp ? page_of(s, c.b, i) : -1;
        c.fresh = true;
      }
      const int src = pg - c.first_page;
      const int id = max(0, __shfl_sync(0xffffffffu, c.page_lane, src));
      if (lane == 0) {
        const int row = (id * a.Hkv + c.h) * s.page + (c.j & ((1 << lg_tp) - 1)) * 32;
        mbar_expect_tx(bar, SLOT);
        tma_load_2d(dst, &map_k, 0, row, bar);
        tma_load_2d(dst + HALF_SLOT, &map_v, 0, row, bar);
      }
      if (c.fresh) {                                            // (the copies need not wait for the scales)
        c.fresh = false;
        c.ks_lane = c.vs_lane = NAN;                            // a page outside the pool makes its rows NaN
        if (c.page_lane >= 0) {
          const size_t ph = (size_t)c.page_lane * a.Hkv + c.h;
          c.ks_lane = bf16_bits_to_f32(__ldg(a.k_scale + ph));
          c.vs_lane = bf16_bits_to_f32(__ldg(a.v_scale + ph));
        }
      }
      const float ks = __shfl_sync(0xffffffffu, c.ks_lane, src), vs = __shfl_sync(0xffffffffu, c.vs_lane, src);
      if (lane == 0) s_scale[warp * PA_STAGES + slot] = make_float2(ks, vs);
    } else if (lane == 0) {
      const int row = (c.b * a.Hkv + c.h) * s.page + (c.j - c.page_tiles) * 16;
      mbar_expect_tx(bar, SLOT);
#pragma unroll
      for (int y = 0; y < D / 64; ++y) {
        tma_load_2d(dst + y * 2048, &map_kt, 64 * y, row, bar);
        tma_load_2d(dst + HALF_SLOT + y * 2048, &map_vt, 64 * y, row, bar);
      }
    }
    __syncwarp();
    // on to the next tile
    ++c.x;
    if (++c.j == c.tiles) {
      c.j = 0;
      c.first_page = -64;
      if (++c.rb == c.row_blocks) {
        c.rb = 0;
        ++c.h;
      }
      if (c.x == c.end && c.x < x1) enter(c.x);
    }
  };
  c.x = x0;
  enter(x0);
  const int total = x1 - x0;
  int issued = 0;
  for (; issued < min(PA_STAGES, total); ++issued) issue(issued);

  // ---- the products
  const float scale_log2 = 1.4426950408889634f * rsqrtf((float)D);
  int k = 0;
  bool ok = true;
  int x = x0;
  int b = seq_at(x0);
  while (x < x1) {
    while (x >= s_base[b + 1].tile) ++b;
    const Seq q = seq_of(s, b);
    const Shape sh = shape_of(q, s.page, p.G, RB);
    const int per = sh.page_tiles + sh.tail_tiles, in = x - s_base[b].tile, item = in / per;
    const int h = item / sh.row_blocks, rb = item - h * sh.row_blocks;
    const int j0 = in - item * per;
    const bool tail = j0 >= sh.page_tiles;
    const int j1 = min(tail ? per : sh.page_tiles, j0 + (x1 - x));           // this record's tiles of the item
    const int rows = min(RB, q.n * p.G - rb * RB), seg = x;     // seg: the piece's first tile

    // query row r of the item: token r / G, head h G + r % G
    auto row_of = [&](int r, int& tok) {
      const int gr = rb * RB + r;
      tok = gr / p.G;
      return a.q + (q.row0 + tok) * a.qs + (size_t)(h * p.G + gr - tok * p.G) * D;
    };
    // B operands: column g is query row 8 nb + g.  For codes: in fp16, times the power of two that brings the row's largest
    // magnitude near 1 (the accumulator takes it off again); the channels in the order in which codes lie in a word.
    uint32_t qf[NB][KS][2];
    float back[NB][2];                                          // accumulator -> logit in powers of two, columns 2t, 2t + 1
    float qsum[NB][2];                                          // int8: 128 times the sum of the column's operands
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int r = 8 * nb + g;
      int tok = 0;
      const uint16_t* src = r < rows ? row_of(r, tok) : nullptr;
      if (tail) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            qf[nb][ks][i] = src ? __ldg(reinterpret_cast<const uint32_t*>(src + 16 * ks + 8 * i + 2 * t)) : 0u;
        back[nb][0] = back[nb][1] = scale_log2;
        qsum[nb][0] = qsum[nb][1] = 0.f;
      } else {
        // lane t of a row has channels 64 cb + 16 t .. + 15
        uint4 v[D / 64][2];
        uint32_t m = 0u;
#pragma unroll
        for (int cb = 0; cb < D / 64; ++cb)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            v[cb][i] = src ? __ldg(reinterpret_cast<const uint4*>(src + 64 * cb + 16 * t + 8 * i)) : make_uint4(0u, 0u, 0u, 0u);
            m = max(m, max(max(max(v[cb][i].x & 0x7fffu, v[cb][i].x >> 16 & 0x7fffu), max(v[cb][i].y & 0x7fffu, v[cb][i].y >> 16 & 0x7fffu)),
                           max(max(v[cb][i].z & 0x7fffu, v[cb][i].z >> 16 & 0x7fffu), max(v[cb][i].w & 0x7fffu, v[cb][i].w >> 16 & 0x7fffu))));
          }
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const int e = min(max((int)(m >> 7), 1), 253);          // exponent field of the largest magnitude
        const float down = __uint_as_float((uint32_t)(254 - e) << 23), up = __uint_as_float((uint32_t)e << 23);
        float sum = 0.f;
#pragma unroll
        for (int cb = 0; cb < D / 64; ++cb) {
          const uint32_t w[8] = {v[cb][0].x, v[cb][0].y, v[cb][0].z, v[cb][0].w, v[cb][1].x, v[cb][1].y, v[cb][1].z, v[cb][1].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {                         // a word of codes: channels 4i .. 4i + 3, int8 as (0, 2) and (1, 3)
            const float c0 = bf16lo(w[2 * i]) * down, c1 = bf16hi(w[2 * i]) * down, c2 = bf16lo(w[2 * i + 1]) * down, c3 = bf16hi(w[2 * i + 1]) * down;
            const uint32_t lo = FORMAT == QP_INT8 ? pack_half2(c0, c2) : pack_half2(c0, c1), hi = FORMAT == QP_INT8 ? pack_half2(c1, c3) : pack_half2(c2, c3);
            qf[nb][4 * cb + i][0] = lo;
            qf[nb][4 * cb + i][1] = hi;
            if (FORMAT == QP_INT8) {
              const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&lo)), f1 = __half22float2(*reinterpret_cast<const __half2*>(&hi));
              sum += (f0.x + f0.y) + (f1.x + f1.y);
            }
          }
        }
        if (FORMAT == QP_INT8) {
          sum += __shfl_xor_sync(0xffffffffu, sum, 1);
          sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          back[nb][i] = __shfl_sync(0xffffffffu, up, 4 * (2 * t + i)) * scale_log2 * kCodeUnit<FORMAT>;
          qsum[nb][i] = FORMAT == QP_INT8 ? __shfl_sync(0xffffffffu, sum, 4 * (2 * t + i)) * (128.f / kCodeUnit<FORMAT>) : 0.f;
        }
      }
    }
    // positions that the columns' rows see: below lim
    int lim[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int tok = 0;
        const int r = 8 * nb + 2 * t + i;
        if (r < rows) row_of(r, tok); else tok = q.n - 1;
        lim[nb][i] = q.len + tok + 1;
      }

    float acc[NB][KS][4], l[NB][2], m_run[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[nb][ks][i] = 0.f;
      l[nb][0] = l[nb][1] = 0.f;
      m_run[nb][0] = m_run[nb][1] = -INFINITY;
    }
    // a new reference for the columns whose logits exceed the old one by more than 2^4 (or that have none yet)
    auto renew = [&](int nb, float mx0, float mx1) {
      if (!__any_sync(0xffffffffu, mx0 > m_run[nb][0] + PA_SLACK || mx1 > m_run[nb][1] + PA_SLACK)) return;
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, o));
        mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, o));
      }
      const float n0 = mx0 > m_run[nb][0] + PA_SLACK ? mx0 : m_run[nb][0], n1 = mx1 > m_run[nb][1] + PA_SLACK ? mx1 : m_run[nb][1];
      const float f0 = n0 == m_run[nb][0] ? 1.f : ex2a(m_run[nb][0] - n0), f1 = n1 == m_run[nb][1] ? 1.f : ex2a(m_run[nb][1] - n1);
      m_run[nb][0] = n0;
      m_run[nb][1] = n1;
      l[nb][0] *= f0;
      l[nb][1] *= f1;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        acc[nb][ks][0] *= f0; acc[nb][ks][1] *= f1;
        acc[nb][ks][2] *= f0; acc[nb][ks][3] *= f1;
      }
    };

    for (int j = j0; j < j1; ++j, ++k, ++x) {
      const int slot = k % PA_STAGES;
      const uint32_t kt = ring + slot * SLOT, vt = kt + HALF_SLOT;
      ok = ok && mbar_wait_warp(bar0 + 8 * slot, (uint32_t)(k / PA_STAGES) & 1u, &give_up);
      if (!ok) break;
      if (!tail) {
        const float2 sc = s_scale[warp * PA_STAGES + slot];
        const int tok0 = 32 * j;
        float sv[NB][2][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int mb = 0; mb < 2; ++mb)
#pragma unroll
            for (int i = 0; i < 4; ++i) sv[nb][mb][i] = 0.f;
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
          for (int cb = 0; cb < D / 64; ++cb) {
            const int r0 = 16 * mb + token_of<D>(g);
            const uint4 w0 = lds128(kt + swz<D>(r0, 4 * cb + t)), w1 = lds128(kt + swz<D>(r0 + 8, 4 * cb + t));
            const uint32_t u0[4] = {w0.x, w0.y, w0.z, w0.w}, u1[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint2 x0 = key_codes<FORMAT>(u0[i]), x1 = key_codes<FORMAT>(u1[i]);
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) mma_f16_m16n8k16(sv[nb][mb], x0.x, x1.x, x0.y, x1.y, qf[nb][4 * cb + i][0], qf[nb][4 * cb + i][1]);
            }
          }
        uint32_t pb[NB][2][2];                                  // weights as B operands: tokens x columns
        float psum[NB][2];                                      // int8: 128 times their sums
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const float f0 = sc.x * back[nb][0], f1 = sc.x * back[nb][1];
          float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
          for (int mb = 0; mb < 2; ++mb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float v = (sv[nb][mb][i] - (FORMAT == QP_INT8 ? qsum[nb][i & 1] : 0.f)) * ((i & 1) ? f1 : f0);
              if (tok0 + 32 > lim[nb][i & 1]) {
                const int tok = tok0 + 16 * mb + 8 * (i >> 1) + token_of<D>(g);
                if (tok >= lim[nb][i & 1]) v = -INFINITY;
              }
              sv[nb][mb][i] = v;
              if (i & 1) mx1 = fmaxf(mx1, v); else mx0 = fmaxf(mx0, v);
            }
          renew(nb, mx0, mx1);
          const float n0 = PA_HEAD - (m_run[nb][0] == -INFINITY ? 0.f : m_run[nb][0]), n1 = PA_HEAD - (m_run[nb][1] == -INFINITY ? 0.f : m_run[nb][1]);
#pragma unroll
          for (int mb = 0; mb < 2; ++mb)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              pb[nb][mb][i] = movmatrix(pack_half2(ex2a(sv[nb][mb][2 * i] + n0), ex2a(sv[nb][mb][2 * i + 1] + n1)));
          // their sums, every row of a product with ones: as the product with the values has them
          float one[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int mb = 0; mb < 2; ++mb) mma_f16_m16n8k16(one, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, pb[nb][mb][0], pb[nb][mb][1]);
          l[nb][0] += one[0];
          l[nb][1] += one[1];
          psum[nb][0] = one[0] * (128.f / kCodeUnit<FORMAT>);
          psum[nb][1] = one[1] * (128.f / kCodeUnit<FORMAT>);
        }
        const float fv = sc.y * kCodeUnit<FORMAT>;
        const int li = lane & 7, lm = lane >> 3;                // row of an 8 x 8 matrix, matrix
        const int vr = 8 * lm + token_of<D>(li);
#pragma unroll
        for (int ch = 0; ch < KS; ++ch) {
          uint32_t w0, w1, w2, w3;
          ldmatrix_x4_trans(w0, w1, w2, w3, vt + swz<D>(vr, ch));
          const uint2 v0 = value_codes<FORMAT>(w0), v1 = value_codes<FORMAT>(w1), v2 = value_codes<FORMAT>(w2), v3 = value_codes<FORMAT>(w3);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float o[4] = {0.f, 0.f, 0.f, 0.f};
            mma_f16_m16n8k16(o, v0.x, v0.y, v1.x, v1.y, pb[nb][0][0], pb[nb][0][1]);
            mma_f16_m16n8k16(o, v2.x, v2.y, v3.x, v3.y, pb[nb][1][0], pb[nb][1][1]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              acc[nb][ch][i] = fmaf(FORMAT == QP_INT8 ? o[i] - psum[nb][i & 1] : o[i], fv, acc[nb][ch][i]);
          }
        }
      } else {
        const int tok0 = (q.len + q.n) / s.page * s.page + 16 * (j - sh.page_tiles), left = q.len + q.n - tok0;
        const int lr = lane & 15, lc = lane >> 4;               // ldmatrix: row, chunk of the pair
        float sv[NB][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 4; ++i) sv[nb][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          uint32_t w[4];
          ldmatrix_x4(w[0], w[1], w[2], w[3], kt + (ks >> 2) * 2048 + swz<128>(lr, 2 * (ks & 3) + lc));
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) mma_bf16_m16n8k16(sv[nb], w, qf[nb][ks][0], qf[nb][ks][1]);
        }
        uint32_t ph[NB][2], pl[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = sv[nb][i] * scale_log2;
            if (tok0 + 8 * (i >> 1) + g >= lim[nb][i & 1]) v = -INFINITY;
            sv[nb][i] = v;
            if (i & 1) mx1 = fmaxf(mx1, v); else mx0 = fmaxf(mx0, v);
          }
          renew(nb, mx0, mx1);
          const float n0 = PA_HEAD - (m_run[nb][0] == -INFINITY ? 0.f : m_run[nb][0]), n1 = PA_HEAD - (m_run[nb][1] == -INFINITY ? 0.f : m_run[nb][1]);
          float one[4] = {0.f, 0.f, 0.f, 0.f};
          const uint32_t ones[4] = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float e0 = ex2a(sv[nb][2 * i] + n0), e1 = ex2a(sv[nb][2 * i + 1] + n1);
            const uint32_t hi = pack_bf16x2(e0, e1), lo = pack_bf16x2(e0 - bf16lo(hi), e1 - bf16hi(hi));
            ph[nb][i] = movmatrix(hi);
            pl[nb][i] = movmatrix(lo);
          }
          mma_bf16_m16n8k16(one, ones, ph[nb][0], ph[nb][1]);
          mma_bf16_m16n8k16(one, ones, pl[nb][0], pl[nb][1]);
          l[nb][0] += one[0];
          l[nb][1] += one[1];
        }
        // rows behind the last token may hold anything
        const uint32_t v0 = (2 * t < left ? 0xffffu : 0u) | (2 * t + 1 < left ? 0xffff0000u : 0u);
        const uint32_t v1 = (2 * t + 8 < left ? 0xffffu : 0u) | (2 * t + 9 < left ? 0xffff0000u : 0u);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          // matrices: tokens 0-7 and 8-15 of channels 16 ks .. + 7, the same of the next 8 channels
          uint32_t w[4];
          ldmatrix_x4_trans(w[0], w[2], w[1], w[3], vt + (ks >> 2) * 2048 + swz<128>(lr, 2 * (ks & 3) + lc));
          w[0] &= v0; w[1] &= v0; w[2] &= v1; w[3] &= v1;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            mma_bf16_m16n8k16(acc[nb][ks], w, ph[nb][0], ph[nb][1]);
            mma_bf16_m16n8k16(acc[nb][ks], w, pl[nb][0], pl[nb][1]);
          }
        }
      }
      __syncwarp();
      if (issued < total) issue(issued++);
    }
#ifdef QP_CHECKED
    const bool lost = (int)blockIdx.x == g_give_up;
#else
    constexpr bool lost = false;
#endif
    if (!ok || lost) {                                          // what is lost, here and in the rest of the run, shows as NaN
      x = seg + (j1 - j0);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) { m_run[nb][0] = m_run[nb][1] = 0.f; l[nb][0] = l[nb][1] = NAN; }
    }

    // ---- the record
    const int slot = 2 * (s_base[b].item + item) + (tail ? 1 : 0) + worker;
    float* rec = p.rec + (size_t)slot * RB * D;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = 8 * nb + 2 * t + i;
        if (r >= rows) continue;
        float* o = rec + (size_t)r * D;
        // (a sum that is no number has to be looked at, whatever was made of the maximum)
        if (g == 0) p.rec_ml[(size_t)slot * RB + r] = make_float2(l[nb][i] == l[nb][i] ? m_run[nb][i] : 0.f, l[nb][i]);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          if (tail) {
            o[16 * ks + g] = acc[nb][ks][i];
            o[16 * ks + 8 + g] = acc[nb][ks][2 + i];
          } else {
            *reinterpret_cast<float2*>(o + 16 * ks + 2 * g) = make_float2(acc[nb][ks][i], acc[nb][ks][2 + i]);
          }
        }
      }
    }
  }
  if (!ok) {
    give_up = 1;
    // the copies still on their way land in this block's shared memory: wait (bounded) for them before it is given up
    for (int i = k; i < issued; ++i)
      for (uint32_t y = 0; y < TC_SPIN_LIMIT; ++y)
        if (mbar_try_wait(bar0 + 8 * (i % PA_STAGES), (uint32_t)(i / PA_STAGES) & 1u)) break;
  }
}

// out from the records, in their order: WPR warps for a query row of a sequence, each with four records on their way at a time.  A
// block is 8 warps: one row where there are few (and so many records for each), else 8 rows.
constexpr int PM_WARPS = 8, PM_BATCH = 4;
template <int D, int WPR>
__global__ void __launch_bounds__(PM_WARPS * 32)
paged_merge_kernel(const __grid_constant__ PagedLaunch p) {
  __shared__ float s_m[PM_WARPS], s_l[PM_WARPS];
  __shared__ float s_o[WPR > 1 ? PM_WARPS : 1][D];
  chain_enter();
  const PagedAttnArgs& a = p.a;
  const StepView& s = a.s;
  const int warp = WPR > 1 ? threadIdx.x >> 5 : 0, lane = threadIdx.x & 31;
  const int row0 = WPR > 1 ? blockIdx.x : blockIdx.x * PM_WARPS + (threadIdx.x >> 5);
  const int b = blockIdx.y, tok = row0 / a.Hq, head = row0 - tok * a.Hq;
  const SeqBase at = p.base[b];
  const int T = p.base[s.n_seqs].tile;
  const Seq q = seq_of(s, b);
  if (tok >= q.n || T == 0) return;
  const Shape sh = shape_of(q, s.page, p.G, p.RB);
  const int W = workers_of(p, T), per = sh.page_tiles + sh.tail_tiles;
  const int h = head / p.G, gr = tok * p.G + head - h * p.G, rb = gr / p.RB, r = gr - rb * p.RB, item = h * sh.row_blocks + rb;
  const int x = at.tile + item * per, slot0 = 2 * (at.item + item);
  // workers of the pages' tiles and of the waiting rows': of the first and the last of each
  const int mine = owner_of(max(0, x + (lane == 0 ? 0 : lane == 1 ? sh.page_tiles - 1 : lane == 2 ? sh.page_tiles : per - 1)), T, W);
  const int w0 = __shfl_sync(0xffffffffu, mine, 0), w1 = __shfl_sync(0xffffffffu, mine, 2);
  const int n0 = sh.page_tiles ? __shfl_sync(0xffffffffu, mine, 1) - w0 + 1 : 0, n1 = sh.tail_tiles ? __shfl_sync(0xffffffffu, mine, 3) - w1 + 1 : 0;
  constexpr int V = D / 32;                                     // channels of a lane
  float M = -INFINITY, L = 0.f, o[V];
#pragma unroll
  for (int i = 0; i < V; ++i) o[i] = 0.f;
  for (int k0 = warp; k0 < n0 + n1; k0 += WPR * PM_BATCH) {
    float2 ml[PM_BATCH];
    float v[PM_BATCH][V];
#pragma unroll
    for (int j = 0; j < PM_BATCH; ++j) {
      const int k = k0 + j * WPR;
      ml[j] = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int i = 0; i < V; ++i) v[j][i] = 0.f;
      if (k < n0 + n1) {
        const size_t row = (size_t)(k < n0 ? slot0 + w0 + k : slot0 + 1 + w1 + k - n0) * p.RB + r;
        ml[j] = p.rec_ml[row];
        const float* src = p.rec + row * D + V * lane;
        if constexpr (V == 4) {
          const float4 f = *reinterpret_cast<const float4*>(src);
          v[j][0] = f.x; v[j][1] = f.y; v[j][2] = f.z; v[j][3] = f.w;
        } else {
          const float2 f = *reinterpret_cast<const float2*>(src);
          v[j][0] = f.x; v[j][1] = f.y;
        }
      }
    }
    float n = M;
#pragma unroll
    for (int j = 0; j < PM_BATCH; ++j) n = fmaxf(n, ml[j].x);
    if (n == -INFINITY) continue;                               // nothing seen
    const float f = M == -INFINITY ? 0.f : ex2a(M - n);
    M = n;
    L *= f;
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] *= f;
#pragma unroll
    for (int j = 0; j < PM_BATCH; ++j) {
      const float e = ml[j].x == -INFINITY ? 0.f : ex2a(ml[j].x - n);
      if (ml[j].x == -INFINITY) continue;
      L = fmaf(ml[j].y, e, L);
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = fmaf(v[j][i], e, o[i]);
    }
  }
  uint16_t* out = a.out + ((size_t)(q.row0 + tok) * a.Hq + head) * D;
  if constexpr (WPR == 1) {
    const float inv = __fdiv_rn(1.f, L);
    if constexpr (V == 4)
      *reinterpret_cast<uint2*>(out + 4 * lane) = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
    else
      *reinterpret_cast<uint32_t*>(out + 2 * lane) = pack_bf16x2(o[0] * inv, o[1] * inv);
    return;
  }
  if (lane == 0) { s_m[warp] = M; s_l[warp] = L; }
#pragma unroll
  for (int i = 0; i < V; ++i) s_o[warp][V * lane + i] = o[i];
  __syncthreads();
  const int d = threadIdx.x;
  if (d >= D) return;
  float m = s_m[0];
#pragma unroll
  for (int w = 1; w < PM_WARPS; ++w) m = fmaxf(m, s_m[w]);
  float l = 0.f, acc = 0.f;
#pragma unroll
  for (int w = 0; w < PM_WARPS; ++w) {
    const float e = s_m[w] == -INFINITY ? 0.f : ex2a(s_m[w] - m);
    l += s_l[w] * e;
    acc += s_o[w][d] * e;
  }
  const __nv_bfloat16 v = __float2bfloat16_rn(__fdiv_rn(acc, l));
  out[d] = *reinterpret_cast<const uint16_t*>(&v);
}

// more query rows per KV head than the products here are made for
bool many_rows(int max_new, int G) { return (long long)max_new * G > 32; }
// (17 to 24 rows at once rather than in two: 5 tokens x 4 heads of 16 sequences of 3000 to 4100, 51.9 us against 53.2)
int rows_of(int max_new, int G) { return max_new * G <= 8 ? 8 : max_new * G > 16 && max_new * G <= 24 ? 24 : 16; }

struct Carve {
  size_t base, ml, rec, total;
  int items;
};
Carve carve(int n_seqs, int n_tokens, int max_new, int Hq, int Hkv, int D) {
  const int G = Hq / Hkv, RB = rows_of(max_new, G);
  const size_t items = Hkv * ((size_t)n_tokens * G / RB + n_seqs), slots = 2 * items + PA_WORKERS;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  Carve c;
  c.items = (int)items;
  c.base = 0;
  c.ml = up((size_t)(n_seqs + 1) * sizeof(SeqBase));
  c.rec = c.ml + up(slots * RB * sizeof(float2));
  c.total = c.rec + slots * RB * D * sizeof(float);
  return c;
}

// rows of `row_bytes` bytes as a [rows x row_bytes] matrix, boxes of box_rows x box_bytes
cudaError_t byte_map(CUtensorMap* map, const void* base, size_t rows, int row_bytes, int box_rows, int box_bytes) {
  EncodeTiledFn enc = encode_tiled();
  if (!enc) return cudaErrorNotSupported;
  const cuuint64_t dims[2] = {(cuuint64_t)row_bytes / 2, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)row_bytes};
  const cuuint32_t box[2] = {(cuuint32_t)box_bytes / 2, (cuuint32_t)box_rows}, elem[2] = {1, 1};
  const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         box_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int FORMAT, int D, int NB, int BUSY>
cudaError_t launch_decode_t(const PagedLaunch& p, const CUtensorMap (&m)[4], cudaStream_t st) {
  static unsigned char done[64];
  constexpr size_t smem = pa_warps(NB, BUSY) * pa_stages(NB, BUSY) * 64 * D + 1024;
  auto kernel = paged_decode_kernel<FORMAT, D, NB, BUSY>;
  cudaError_t e = allow_smem(kernel, smem, done);
  if (e != cudaSuccess) return e;
  e = launch_chained(kernel, dim3(PA_SMS), dim3(pa_warps(NB, BUSY) * 32), smem, st, p, m[0], m[1], m[2], m[3]);
  if (e != cudaSuccess) return e;
  const unsigned rows = (unsigned)p.a.s.max_new * p.a.Hq;
  if (rows * p.a.s.n_seqs <= 8 * PA_SMS) return launch_chained(paged_merge_kernel<D, PM_WARPS>, dim3(rows, p.a.s.n_seqs), dim3(PM_WARPS * 32), 0, st, p);
  return launch_chained(paged_merge_kernel<D, 1>, dim3((rows + PM_WARPS - 1) / PM_WARPS, p.a.s.n_seqs), dim3(PM_WARPS * 32), 0, st, p);
}

}  // namespace

#ifdef QP_CHECKED
cudaError_t paged_attn_check_read(unsigned int (&out)[4]) { return checked::read_and_clear(out); }
cudaError_t paged_attn_give_up(int block) { return cudaMemcpyToSymbol(g_give_up, &block, sizeof(block)); }
#endif

bool paged_attn_fits(int n_seqs, int n_tokens, int max_new, int Hq, int Hkv, long long most_len) {
  if (many_rows(max_new, Hq / Hkv)) return paged_chunk_fits(n_seqs, n_tokens, Hq, Hkv, most_len);
  const long long G = Hq / Hkv, items = Hkv * (n_tokens * G / rows_of(max_new, (int)G) + n_seqs);
  return items < 0x7fffffffLL / (most_len / 32 + 8);
}
size_t paged_attn_workspace(int n_seqs, int n_tokens, int max_new, int Hq, int Hkv, int D) {
  if (many_rows(max_new, Hq / Hkv)) return paged_chunk_workspace(n_seqs, n_tokens, Hq, Hkv, D);
  return carve(n_seqs, n_tokens, max_new, Hq, Hkv, D).total;
}

cudaError_t launch_paged_attn(const PagedAttnArgs& a, void* ws, cudaStream_t st) {
  CUtensorMap m[4];
  const size_t rows = (size_t)a.s.n_pages * a.Hkv * a.s.page, tail_rows = (size_t)a.s.n_seqs * a.Hkv * a.s.page;
  cudaError_t e = byte_map(&m[0], a.kc, rows, a.D, 32, a.D);
  if (e == cudaSuccess) e = byte_map(&m[1], a.vc, rows, a.D, 32, a.D);
  if (e != cudaSuccess) return e;
  if (many_rows(a.s.max_new, a.Hq / a.Hkv)) return launch_paged_chunk(a, ws, m[0], m[1], st);
  PagedLaunch p{};
  p.a = a;
  p.G = a.Hq / a.Hkv;
  p.RB = rows_of(a.s.max_new, p.G);
  const bool busy = (long long)a.s.n_seqs * a.Hkv >= 64;
  p.n_workers = PA_SMS * pa_warps(p.RB / 8, busy);
  p.min_tiles = 2;
  const Carve c = carve(a.s.n_seqs, a.s.n_tokens, a.s.max_new, a.Hq, a.Hkv, a.D);
  p.max_items = c.items;
  char* w = static_cast<char*>(ws);
  p.base = reinterpret_cast<SeqBase*>(w + c.base);
  p.rec_ml = reinterpret_cast<float2*>(w + c.ml);
  p.rec = reinterpret_cast<float*>(w + c.rec);
  e = byte_map(&m[2], a.k_tail, tail_rows, 2 * a.D, 16, 128);
  if (e == cudaSuccess) e = byte_map(&m[3], a.v_tail, tail_rows, 2 * a.D, 16, 128);
  if (e != cudaSuccess) return e;
#define QP_PAGED(F, DD)                                             \
  return p.RB == 8    ? busy ? launch_decode_t<F, DD, 1, 1>(p, m, st) : launch_decode_t<F, DD, 1, 0>(p, m, st) \
         : p.RB == 16 ? busy ? launch_decode_t<F, DD, 2, DD == 128>(p, m, st) : launch_decode_t<F, DD, 2, 0>(p, m, st) \
                      : launch_decode_t<F, DD, 3, 0>(p, m, st)
  if (a.format == QP_E4M3) {
    if (a.D == 128) QP_PAGED(QP_E4M3, 128);
    QP_PAGED(QP_E4M3, 64);
  }
  if (a.D == 128) QP_PAGED(QP_INT8, 128);
  QP_PAGED(QP_INT8, 64);
#undef QP_PAGED
}

}  // namespace qp
