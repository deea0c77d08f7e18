// Decode attention that accumulates its softmax weights (qp_decode_attn_weights).
//
//   out[h] = sum_t p[h,t] V'[t],   W[t] += sum_h p[h,t],   p[h,t] = 2^(x[h,t] - M[h]) / Z[h],   x = q.K' log2(e) / sqrt(D)
//
// A token's weight needs the normaliser over all tokens, the output does not: the logits are kept (G floats per token, against
// 2 D B / 8 bytes of cache) until the head's statistics are known.  One thread-block cluster per (batch, KV head) makes this one
// launch: CTA r streams a contiguous run of 32-token tiles with one pass over keys and values, leaves (max, sum, accumulators)
// in its shared memory, the cluster exchanges them through distributed shared memory, and every CTA then turns its own logits
// into weights and writes its slice of the output.  Bound: the packed bytes from HBM; the logits stay in shared memory, or for
// very long runs in the caller's workspace (L2).
//
// The weights are results of their own, so logits, maxima and sums are held in 32 bits: queries enter the tensor cores unscaled,
// codes are integers, and scales, zero points and log2(e)/sqrt(D) (by the approximate reciprocal root, 2 ulp) are applied to
// 32-bit accumulators.  At 16 bit every factor of a logit is exact; in packed caches a query channel is a bf16 value times 2^-p,
// p <= 8 - B, in f16: exact from 2^(p-17) on, below that off by at most 2^(p-25), at 2 bit 2^-19.  Only the second product, whose
// result is rounded to bf16, uses weights rounded to 16 bits: bf16 in 16-bit caches, like their values (2^-8 of a weight), f16 in
// packed ones (2^-11, and 2^-11 for the product with the scale).
//
// Measured in a replayed graph: 8192 tokens x 64 KV heads at 4 bit 25.2 us = 3.5 TB/s (the stream 17 us of it, exchange and weights
// 5), 5001 x 32 KV heads of eight query heads at 16 bit 20.8 us = 4.0 TB/s, 512 tokens x 8 KV heads at 16 bit 5.5 us.
//
// Per-token caches (B = 2, 4, 8; both matrices [token][D] with groups of g channels): a 16-bit lane holding a small integer c
// is the f16 number c * 2^-24, so masked words are MMA operands; see decode_weights_packed_kernel.
#include <cooperative_groups.h>

#include <algorithm>

#include "qp_cluster.cuh"
#include "qp_mma.cuh"

namespace qp {

namespace {

namespace cg = cooperative_groups;

constexpr int DW_WARPS = 4, DW_THREADS = DW_WARPS * 32, DW_MAX_CLUSTER = 16;
constexpr int DW_LOGIT_BYTES = 24576;  // of shared memory; runs with more logits keep them in the workspace

struct DwArgs {
  DecLayer ly;
  int Bt, Hq, Hkv, group, cluster;
  float* weights;
  float* logits;                         // workspace [BH, G, n32], null: shared memory holds them
  int n32;                               // tokens rounded up to whole tiles
};

// ---- what both kernels do around their streams

// this CTA's run of tiles
__device__ __forceinline__ void dw_run(const DwArgs& a, int rank, int& lo, int& hi) {
  const int tiles = a.n32 / 32;
  lo = (int)((long long)tiles * rank / a.cluster);
  hi = (int)((long long)tiles * (rank + 1) / a.cluster);
}

// After a __syncthreads: warps' partial results s_acc [warp][8][D], s_m, s_l [warp][8] -> this CTA's (in s_out [8][D], s_ml [8][2]),
// -> across the cluster -> weights of this CTA's tokens and a slice of the output.  lg: logits of this CTA's run, head h at
// lg + h * stride, first token at index 0.
template <int D, int WARPS>
__device__ __forceinline__ void dw_finish(const DwArgs& a, int bh, int G, int tok_lo, int tok_hi, const float* s_acc, const float* s_m,
                                          const float* s_l, float* s_out, float2* s_ml, const float* lg, size_t stride) {
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, rank = (int)cluster.block_rank(), C = a.cluster;
  for (int idx = tid; idx < G * D; idx += WARPS * 32) {
    const int h = idx / D, d = idx % D;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) M = fmaxf(M, s_m[w * 8 + h]);
    float Z = 0.f, A = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float mw = s_m[w * 8 + h];
      if (mw != -INFINITY) {
        const float f = ex2(mw - M);
        Z = fmaf(s_l[w * 8 + h], f, Z);
        A = fmaf(s_acc[(w * 8 + h) * D + d], f, A);
      }
    }
    s_out[idx] = A;
    if (d == 0) s_ml[h] = make_float2(M, Z);
  }
  __syncthreads();
  // the statistics are handed to every CTA before the barrier (a read after it would be a round trip of a thousand clocks);
  // the wait is for the arrival at the kernel's start: all CTAs of the cluster are running
  __shared__ float2 s_all[DW_MAX_CLUSTER][8];
  cluster.barrier_wait();
  if (tid < 8 * C && (tid & 7) < G) cluster.map_shared_rank(&s_all[0][0], tid >> 3)[rank * 8 + (tid & 7)] = s_ml[tid & 7];
  cluster.sync();
  // head statistics of the whole cluster
  __shared__ float2 s_head[8];           // (M, 1 / Z)
  __shared__ float s_f[DW_MAX_CLUSTER][8];
  if (tid < G) {
    float2 v[DW_MAX_CLUSTER];
    float M = -INFINITY, Z = 0.f;
#pragma unroll
    for (int r = 0; r < DW_MAX_CLUSTER; ++r) {
      if (r < C) v[r] = s_all[r][tid];
      if (r < C) M = fmaxf(M, v[r].x);
    }
#pragma unroll
    for (int r = 0; r < DW_MAX_CLUSTER; ++r)
      if (r < C) {
        const float f = v[r].x == -INFINITY ? 0.f : ex2(v[r].x - M);
        Z = fmaf(v[r].y, f, Z);
        s_f[r][tid] = f;
      }
    s_head[tid] = make_float2(M, __fdiv_rn(1.0f, Z));
  }
  __syncthreads();
  // the output's slice of this CTA, ranks in order
  const int per = (G * D + C - 1) / C, o_hi = min(G * D, (rank + 1) * per);
  for (int idx = rank * per + tid; idx < o_hi; idx += WARPS * 32) {
    const int h = idx / D;
    float A = 0.f;
    float v[DW_MAX_CLUSTER];
#pragma unroll
    for (int r = 0; r < DW_MAX_CLUSTER; ++r) v[r] = r < C ? cluster.map_shared_rank(s_out, r)[idx] : 0.f;
#pragma unroll
    for (int r = 0; r < DW_MAX_CLUSTER; ++r) A = r < C ? fmaf(v[r], s_f[r][h], A) : A;
    static_cast<bf16*>(a.ly.out)[(size_t)bh * G * D + idx] = __float2bfloat16_rn(A * s_head[h].y);
  }
  __syncwarp();
  cluster.barrier_arrive();              // done with the others' shared memory
  float* w = a.weights + (size_t)bh * a.ly.ns;
  const bool quads = (a.ly.ns & 3) == 0; // rows of weights begin on 16 bytes
  for (int t = tok_lo + 4 * tid; t < tok_hi; t += 4 * WARPS * 32) {      // all heads' logits of four tokens in flight
    float4 x[8];
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < 8; ++h)
      if (h < G) x[h] = *reinterpret_cast<const float4*>(lg + h * stride + (t - tok_lo));
#pragma unroll
    for (int h = 0; h < 8; ++h)
      if (h < G) {
        const float M = s_head[h].x, inv = s_head[h].y;
        s[0] = fmaf(ex2(x[h].x - M), inv, s[0]);
        s[1] = fmaf(ex2(x[h].y - M), inv, s[1]);
        s[2] = fmaf(ex2(x[h].z - M), inv, s[2]);
        s[3] = fmaf(ex2(x[h].w - M), inv, s[3]);
      }
    // one addition per token: no order to depend on, nothing to wait for
    if (quads && t + 4 <= tok_hi) {
      asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};\n" ::"l"(w + t), "f"(s[0]), "f"(s[1]), "f"(s[2]), "f"(s[3]) : "memory");
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (t + i < tok_hi) atomicAdd(&w[t + i], s[i]);
    }
  }
  __syncwarp();
  cluster.barrier_wait();                // nobody leaves while another may still read its shared memory
}

// ---- 16-bit caches: query heads as MMA rows, so the weights leave the first product in the layout the second wants.  Eight
// warps that walk over 16 tokens each: the stream is bound by how many warps wait for their own copies and products, not by
// bytes in flight.
constexpr int DW16_STAGES = 3, DW16_WARPS = 8, DW16_THREADS = DW16_WARPS * 32;

template <int D>
constexpr size_t dw16_smem() { return (size_t)DW16_WARPS * DW16_STAGES * 64 * D + DW_LOGIT_BYTES; }

template <int D>
__global__ void __launch_bounds__(DW16_THREADS, 1)
decode_weights16_kernel(const __grid_constant__ DwArgs a) {
  constexpr int CPR = D / 8, KST = D / 16, NJ = D / 8, TILE = 64 * D, VOFF = 32 * D;   // bytes of 16 tokens: keys, then values
  extern __shared__ __align__(128) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int G = a.Hq / a.Hkv, C = a.cluster, bh = blockIdx.x / C, n = a.ly.n;
  int lo, hi;
  dw_run(a, blockIdx.x % C, lo, hi);
  const int tok_lo = lo * 32, tok_hi = min(n, hi * 32);
  float* lg = a.logits ? a.logits + (size_t)bh * G * a.n32 + tok_lo : reinterpret_cast<float*>(smem + DW16_WARPS * DW16_STAGES * TILE);
  const size_t lstride = a.logits ? (size_t)a.n32 : (size_t)((a.n32 / 32 + C - 1) / C * 32);
  cg::this_cluster().barrier_arrive();   // waited for before the first access to another CTA's shared memory
  chain_enter();

  const uint32_t wsm = smem_u32(smem + warp * (DW16_STAGES * TILE));
  // this lane's pieces of a tile: rows tau0 + i * TSTEP (of 16), one 16-byte column
  constexpr int TSTEP = 32 / CPR, NP = 16 / TSTEP;
  const int tau0 = lane / CPR, ch = lane % CPR;
  uint32_t dst[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) dst[i] = (tau0 + i * TSTEP) * (2 * D) + ((ch ^ ((tau0 + i * TSTEP) & 7)) << 4);
  int tok = tok_lo + warp * 16;                                 // first token of the next tile to fetch
  const size_t row0 = ((size_t)bh * a.ly.ns + tok + tau0) * (D * 2) + ch * 16;
  const unsigned char* gk = static_cast<const unsigned char*>(a.ly.kc) + row0;
  const unsigned char* gv = static_cast<const unsigned char*>(a.ly.vc) + row0;
  auto issue = [&](uint32_t sb) {
    if (tok + 16 <= n) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        cp_async16(sb + dst[i], gk + i * TSTEP * (D * 2));
        cp_async16(sb + VOFF + dst[i], gv + i * TSTEP * (D * 2));
      }
    } else {                                                    // rows behind the last token are zeros, whatever the array holds
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const bool ok = tok + tau0 + i * TSTEP < n;
        cp_async16_zfill(sb + dst[i], ok ? gk + i * TSTEP * (D * 2) : static_cast<const unsigned char*>(a.ly.kc), ok);
        cp_async16_zfill(sb + VOFF + dst[i], ok ? gv + i * TSTEP * (D * 2) : static_cast<const unsigned char*>(a.ly.vc), ok);
      }
    }
    tok += DW16_WARPS * 16;
    gk += DW16_WARPS * 16 * (D * 2);
    gv += DW16_WARPS * 16 * (D * 2);
  };
  // tiles of 16 tokens with at least one token: every one of them has a finite maximum
  const int n_tiles = (tok_hi - tok_lo + 15) / 16, n_my = max(0, (n_tiles - warp + DW16_WARPS - 1) / DW16_WARPS);
#pragma unroll
  for (int s = 0; s < DW16_STAGES - 1; ++s) {
    if (s < n_my) issue(wsm + s * TILE);
    cp_async_commit();
  }
  uint32_t qa[KST][2];
  {
    const uint16_t* q = static_cast<const uint16_t*>(a.ly.q) + ((size_t)bh * G + g) * D;
#pragma unroll
    for (int c = 0; c < KST; ++c) {
      qa[c][0] = g < G ? *reinterpret_cast<const uint32_t*>(q + 16 * c + 2 * t) : 0u;
      qa[c][1] = g < G ? *reinterpret_cast<const uint32_t*>(q + 16 * c + 8 + 2 * t) : 0u;
    }
  }
  const float scale_log2 = 1.4426950408889634f * rsqrtf((float)D);
  const int lrow = lane & 7, lsel = lane >> 3;
  float m_run = -INFINITY, l_run = 0.f, acc[NJ][4];             // head g (m replicated over t)
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int x = 0; x < 4; ++x) acc[j][x] = 0.f;

  uint32_t sb = wsm, sb_copy = wsm + (DW16_STAGES - 1) * TILE;
  for (int it = 0; it < n_my; ++it) {
    __syncwarp();
    if (it + DW16_STAGES - 1 < n_my) issue(sb_copy);
    cp_async_commit();
    cp_async_wait<DW16_STAGES - 1>();
    __syncwarp();
    const int tok0 = tok_lo + (warp + DW16_WARPS * it) * 16;
    float sc[2][4];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
      const int tau = 8 * nt + lrow;
#pragma unroll
      for (int c = 0; c < KST; c += 2) {
        uint32_t b0, b1, b2, b3;
        ldmatrix_x4(b0, b1, b2, b3, sb + tau * (2 * D) + (((2 * c + lsel) ^ (tau & 7)) << 4));
        mma_bf16_m16n8k16(sc[nt], {qa[c][0], 0u, qa[c][1], 0u}, b0, b1);
        mma_bf16_m16n8k16(sc[nt], {qa[c + 1][0], 0u, qa[c + 1][1], 0u}, b2, b3);
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      const int tk = tok0 + 8 * nt + 2 * t;
      sc[nt][0] = tk < n ? sc[nt][0] * scale_log2 : -INFINITY;
      sc[nt][1] = tk + 1 < n ? sc[nt][1] * scale_log2 : -INFINITY;
      mx = fmaxf(mx, fmaxf(sc[nt][0], sc[nt][1]));
      if (g < G) *reinterpret_cast<float2*>(lg + g * lstride + (tk - tok_lo)) = make_float2(sc[nt][0], sc[nt][1]);
    }
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
    const float mnew = fmaxf(m_run, mx), corr = ex2(m_run - mnew);
    m_run = mnew;
    uint32_t pa[2];
    float sum = 0.f;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
      const float p0 = ex2(sc[nt][0] - mnew), p1 = ex2(sc[nt][1] - mnew);
      sum += p0 + p1;
      pa[nt] = pack_bf16x2(p0, p1);
    }
    l_run = fmaf(l_run, corr, sum);
    if (__any_sync(0xffffffffu, corr != 1.f)) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) { acc[j][0] *= corr; acc[j][1] *= corr; }
    }
#pragma unroll
    for (int j = 0; j < NJ; j += 2) {
      const int tau = 8 * (lsel & 1) + lrow;                    // matrices: tokens 0-7, 8-15 of column block j, then of j + 1
      uint32_t v0, v1, v2, v3;
      ldmatrix_x4_trans(v0, v1, v2, v3, sb + VOFF + tau * (2 * D) + (((j + (lsel >> 1)) ^ (tau & 7)) << 4));
      mma_bf16_m16n8k16(acc[j], {pa[0], 0u, pa[1], 0u}, v0, v1);
      mma_bf16_m16n8k16(acc[j + 1], {pa[0], 0u, pa[1], 0u}, v2, v3);
    }
    sb_copy = sb;
    sb = sb + TILE == wsm + DW16_STAGES * TILE ? wsm : sb + TILE;
  }
  l_run += __shfl_xor_sync(0xffffffffu, l_run, 1);
  l_run += __shfl_xor_sync(0xffffffffu, l_run, 2);
  cp_async_wait<0>();
  __syncthreads();                                              // the stages are idle
  float* s_acc = reinterpret_cast<float*>(smem);                // [warp][8][D]
  float *s_m = s_acc + DW16_WARPS * 8 * D, *s_l = s_m + DW16_WARPS * 8, *s_out = s_l + DW16_WARPS * 8;
  float2* s_ml = reinterpret_cast<float2*>(s_out + 8 * D);
#pragma unroll
  for (int j = 0; j < NJ; ++j)
    *reinterpret_cast<float2*>(s_acc + (warp * 8 + g) * D + 8 * j + 2 * t) = make_float2(acc[j][0], acc[j][1]);
  if (t == 0) { s_m[warp * 8 + g] = m_run; s_l[warp * 8 + g] = l_run; }
  __syncthreads();
  dw_finish<D, DW16_WARPS>(a, bh, G, tok_lo, tok_hi, s_acc, s_m, s_l, s_out, s_ml, lg, lstride);
}

// ---- per-token caches
// Keys, first product (rows = 16 tokens, columns = heads): ldmatrix hands lane (g, t) the 32-bit word t of a 16-byte piece of
// token g: CHW = 32/B channels.  The word's pair f is (field f, field f + CHW/2), 16 bits apart: `word & mask` is an f16 operand
// pair of integers times 2^-24 times 2^(position), pairs beyond the first byte after a shift by 8.  The contraction index is a
// permutation of the channels that the query operand follows; it also carries the factors 2^-(position).
// Values, second product (rows = channels, columns = heads): the transposing ldmatrix hands lane (g, t) the 16-bit unit g of
// tokens 2t and 2t+1: U = 16/B channels, field f of both tokens again by masking.  The scale goes into the weights (per group),
// the zero points are one small product of their own.
// At 2 bits a 16-byte piece is 64 channels: with groups of 32 it holds two, and the operand lanes of the other group are zeroed.
template <int BITS, int D, int GROUP>
struct Pk {
  static constexpr int RB = D * BITS / 8;              // bytes of a token's codes
  static constexpr int NP = RB / 16;                   // 16-byte pieces of them
  static constexpr int NG = D / GROUP;                 // groups per token
  static constexpr int CH = 128 / BITS, CHW = 32 / BITS, U = 16 / BITS;
  static constexpr int SETS = CH > GROUP ? CH / GROUP : 1;      // groups that share a piece
  static constexpr int PPG = CH > GROUP ? 1 : GROUP / CH;       // pieces of a group
  // a 32-token tile in shared memory
  static constexpr int KC = 0, VC = 32 * RB, KS = 64 * RB, MB = 64 * NG, KZ = KS + MB, VS = KZ + MB, VZ = VS + MB, BYTES = VZ + MB;
  // two stages and three blocks per SM (the launch bounds): a third stage or a fourth block cost 4 to 9 % (8192 x 64 heads, 4 bit;
  // a fourth block leaves 128 registers a thread)
  static constexpr int STAGES = 2;
  static constexpr int P_STRIDE = 80, P_BYTES = 8 * P_STRIDE;   // weights of a tile, [head][32 tokens] f16 and a pad
  static constexpr int WARP_BYTES = STAGES * BYTES + P_BYTES;
  static constexpr size_t SMEM = (size_t)DW_WARPS * WARP_BYTES + DW_LOGIT_BYTES;
  // the epilogue's arrays overlay the stages
  static constexpr int EPI = (DW_WARPS * 8 * D + 2 * DW_WARPS * 8 + 8 * D + 16) * 4;
  static constexpr size_t SMEM_ALL = SMEM > (size_t)EPI + DW_LOGIT_BYTES ? SMEM : (size_t)EPI + DW_LOGIT_BYTES;
  static __host__ __device__ constexpr int piece(int tau, int v) {      // conflict-free for both ldmatrix forms
    const int sw = RB == 128 ? tau & 7 : RB == 64 ? (tau >> 1) & 3 : RB == 32 ? (tau >> 2) & 1 : 0;
    return tau * RB + ((v ^ sw) << 4);
  }
};

// N halves from shared memory, aligned to their size, in the widest loads
template <int N>
__device__ __forceinline__ void lds_halves(__half (&h)[N], uint32_t addr) {
  if constexpr (N == 8) {
    *reinterpret_cast<uint4*>(h) = lds128(addr);
  } else if constexpr (N == 4) {
    *reinterpret_cast<uint2*>(h) = lds64(addr);
  } else if constexpr (N == 2) {
    *reinterpret_cast<uint32_t*>(h) = lds32(addr);
  } else {
    unsigned short v;
    asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(v) : "r"(addr));
    h[0] = *reinterpret_cast<const __half*>(&v);
  }
}

__device__ __forceinline__ uint32_t max_half2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.f16x2 %0, %1, %2;\n" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// N halves (1, 2 or 4) from shared memory as a pair with the same maximum
template <int N>
__device__ __forceinline__ uint32_t lds_max_half2(uint32_t addr) {
  __half h[N];
  lds_halves(h, addr);
  if constexpr (N == 1) return (uint32_t)__half_as_ushort(h[0]) * 0x10001u;
  else if constexpr (N == 2) return *reinterpret_cast<const uint32_t*>(h);
  else return max_half2(reinterpret_cast<const uint32_t*>(h)[0], reinterpret_cast<const uint32_t*>(h)[1]);
}

template <int BITS, int D, int GROUP>
__global__ void __launch_bounds__(DW_THREADS, 3)
decode_weights_packed_kernel(const __grid_constant__ DwArgs a) {
  using L = Pk<BITS, D, GROUP>;
  constexpr int NP = L::NP, NG = L::NG, NF = L::CHW / 2;        // NF: operand pairs of a word
  constexpr float C24 = 16777216.0f;
  extern __shared__ __align__(128) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int G = a.Hq / a.Hkv, C = a.cluster, bh = blockIdx.x / C;
  int lo, hi;
  dw_run(a, blockIdx.x % C, lo, hi);
  const int tok_lo = lo * 32, tok_hi = hi * 32;                 // n is a multiple of 32
  float* lg_out = a.logits ? a.logits + (size_t)bh * G * a.n32 + tok_lo : reinterpret_cast<float*>(smem + L::SMEM_ALL - DW_LOGIT_BYTES);
  const size_t lstride = a.logits ? (size_t)a.n32 : (size_t)((a.n32 / 32 + C - 1) / C * 32);
  cg::this_cluster().barrier_arrive();   // waited for before the first access to another CTA's shared memory
  chain_enter();

  const uint32_t wsm = smem_u32(smem + warp * L::WARP_BYTES), sP = wsm + L::STAGES * L::BYTES;
  // copies of a tile: this lane's pieces of both code blocks, and of the four scale / zero arrays; the pointers walk from
  // one tile of this warp to its next, DW_WARPS tiles on
  constexpr int MP = L::MB / 16, MPL = (4 * MP + 31) / 32;      // 16-byte pieces of one such array; pieces of all four per lane
  const size_t row0 = (size_t)bh * a.ly.ns + (size_t)(lo + warp) * 32;
  const unsigned char* gk = static_cast<const unsigned char*>(a.ly.kc) + row0 * L::RB + lane * 16;
  const unsigned char* gv = static_cast<const unsigned char*>(a.ly.vc) + row0 * L::RB + lane * 16;
  const unsigned char* gm[MPL];
  uint32_t cdst[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) cdst[i] = L::piece((lane + 32 * i) / NP, (lane + 32 * i) % NP);
#pragma unroll
  for (int i = 0; i < MPL; ++i) {
    const int c = lane + 32 * i, arr = c / MP;
    const __half* src = arr == 0 ? a.ly.ks : arr == 1 ? a.ly.kz : arr == 2 ? a.ly.vs : a.ly.vz;
    gm[i] = reinterpret_cast<const unsigned char*>(src) + row0 * NG * 2 + (c % MP) * 16;
  }
  auto issue = [&](uint32_t sb) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      cp_async16(sb + L::KC + cdst[i], gk + i * 512);
      cp_async16(sb + L::VC + cdst[i], gv + i * 512);
    }
#pragma unroll
    for (int i = 0; i < MPL; ++i) {
      if (lane + 32 * i < 4 * MP) cp_async16(sb + L::KS + (lane + 32 * i) * 16, gm[i]);   // the arrays lie one behind the other
      gm[i] += DW_WARPS * 64 * NG;
    }
    gk += DW_WARPS * 32 * L::RB;
    gv += DW_WARPS * 32 * L::RB;
  };
  const int n_my = max(0, (hi - lo - warp + DW_WARPS - 1) / DW_WARPS);
#pragma unroll
  for (int s = 0; s < L::STAGES - 1; ++s) {
    if (s < n_my) issue(wsm + s * L::BYTES);
    cp_async_commit();
  }

  // query operands: pair f of word t of piece v, channels v CH + t CHW + f (+ CHW/2), times 2^-(position); head g
  const float scale_log2 = 1.4426950408889634f * rsqrtf((float)D);
  uint32_t qb[NP][NF];
  float qsum[NG][2];                                            // sum of a group's query channels, heads 2t and 2t+1, scaled
  {
    const uint16_t* q = static_cast<const uint16_t*>(a.ly.q) + ((size_t)bh * G + (g < G ? g : 0)) * D;
    float part[NG];
#pragma unroll
    for (int i = 0; i < NG; ++i) part[i] = 0.f;
#pragma unroll
    for (int v = 0; v < NP; ++v)
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        const int d0 = v * L::CH + t * L::CHW + f, d1 = d0 + L::CHW / 2;
        const float x = g < G ? bf16_bits_to_f32(q[d0]) : 0.f, y = g < G ? bf16_bits_to_f32(q[d1]) : 0.f;
        const float down = 1.0f / (float)(1 << ((f * BITS) & 7));
        qb[v][f] = pack_half2(x * down, y * down);
#pragma unroll
        for (int i = 0; i < NG; ++i) part[i] += d0 / GROUP == i ? x + y : 0.f;      // (a word lies in one group)
      }
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      float s = part[i];
      s += __shfl_xor_sync(0xffffffffu, s, 1);
      s += __shfl_xor_sync(0xffffffffu, s, 2);                  // lanes (g, *): head g
      qsum[i][0] = __shfl_sync(0xffffffffu, s, 8 * t) * scale_log2;
      qsum[i][1] = __shfl_sync(0xffffffffu, s, 8 * t + 4) * scale_log2;
    }
  }
  const float kscale = C24 * scale_log2;
  const int tau_ld = 8 * (lane >> 3) + (lane & 7);              // ldmatrix row of this lane

  float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};       // heads 2t, 2t+1 (l: this lane's tokens)
  // Weights and their products with the scales are f16 numbers: the reference is held so low that both use the upper end of f16's
  // range, weights up to 2^top with 2^top times the largest scale at most 2^15.  (With the maximum itself as the reference light
  // tokens of small values were lost: at 8 bit the product of 2^-11 with a scale of 2^-13 is the last place of f16.)  The bound
  // on the scales so far is a power of two from 1 on, so that a reference is hardly ever renewed for its sake: with the largest
  // scale itself 8192 tokens x 64 KV heads took 25.8 us at 4 bit, with the power of two 25.2, without any of it 24.9.
  uint32_t bound2 = 0x3c003c00u;                                // twice; like top the same in the whole warp
  float top = 15.f;
  constexpr int MT = L::U / 2;                                  // products per piece of the value side: two fields each
  float acc[NP][MT][4], acc_z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int v = 0; v < NP; ++v)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[v][mt][e] = 0.f;

  uint32_t sb = wsm, sb_copy = wsm + (L::STAGES - 1) * L::BYTES;
  for (int it = 0; it < n_my; ++it) {
    __syncwarp();
    if (it + L::STAGES - 1 < n_my) issue(sb_copy);
    cp_async_commit();
    cp_async_wait<L::STAGES - 1>();
    __syncwarp();
    const int tok0 = (lo + warp + DW_WARPS * it) * 32;

    // ---- keys: lane (g, t) ends up with tokens g + 8j and heads 2t + e
    float lg[4][2] = {{0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}};
    __half ksh[4][NG], kzh[4][NG];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      lds_halves(ksh[j], sb + L::KS + (g + 8 * j) * NG * 2);
      lds_halves(kzh[j], sb + L::KZ + (g + 8 * j) * NG * 2);
    }
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      float a0[4] = {0.f, 0.f, 0.f, 0.f}, a1[4] = {0.f, 0.f, 0.f, 0.f};         // tokens 0..15, 16..31
#pragma unroll
      for (int pp = 0; pp < L::PPG; ++pp) {
        const int v = L::SETS > 1 ? gi / L::SETS : gi * L::PPG + pp;
        uint32_t r[4];
        ldmatrix_x4(r[0], r[1], r[2], r[3], sb + L::KC + L::piece(tau_ld, v));
        const bool mine = L::SETS == 1 || t / (4 / L::SETS) == gi % L::SETS;    // this lane's word belongs to group gi
#pragma unroll
        for (int f = 0; f < NF; f += 2) {
          uint32_t x[4], y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            constexpr uint32_t ones = (1u << BITS) - 1u;
            const int p0 = f * BITS, p1 = (f + 1) * BITS;
            x[i] = (p0 < 8 ? r[i] : r[i] >> 8) & ((ones | ones << 16) << (p0 & 7));
            y[i] = (p1 < 8 ? r[i] : r[i] >> 8) & ((ones | ones << 16) << (p1 & 7));
          }
          const uint32_t b0 = mine ? qb[v][f] : 0u, b1 = mine ? qb[v][f + 1] : 0u;
          mma_f16_m16n8k16(a0, x[0], x[1], y[0], y[1], b0, b1);
          mma_f16_m16n8k16(a1, x[2], x[3], y[2], y[3], b0, b1);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float s = __half2float(ksh[j][gi]) * kscale, z = __half2float(kzh[j][gi]);
        lg[j][0] = fmaf(s, (j < 2 ? a0 : a1)[2 * (j & 1)], fmaf(z, qsum[gi][0], lg[j][0]));
        lg[j][1] = fmaf(s, (j < 2 ? a0 : a1)[2 * (j & 1) + 1], fmaf(z, qsum[gi][1], lg[j][1]));
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (2 * t + e < G)
#pragma unroll
        for (int j = 0; j < 4; ++j) lg_out[(2 * t + e) * lstride + (tok0 - tok_lo + g + 8 * j)] = lg[j][e];

    // ---- running softmax; the reference is renewed only when a logit exceeds it by more than `top`, and then leaves it 4 to grow
    float over = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j) over = fmaxf(over, fmaxf(lg[j][0] - m_run[0], lg[j][1] - m_run[1]));
    uint32_t scale2 = max_half2(bound2, lds_max_half2<NG>(sb + L::VS + lane * NG * 2));              // with those of token `lane`
    if (__any_sync(0xffffffffu, over > top || scale2 != bound2)) {
      scale2 = max_half2(scale2, scale2 << 16 | scale2 >> 16);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) scale2 = max_half2(scale2, __shfl_xor_sync(0xffffffffu, scale2, o));
      const int e = (int)((scale2 & 0xffffu) + 0x3ffu) >> 10;                    // exponent field of the next power of two
      bound2 = min(e << 10, 0x7bff) * 0x10001u;                                  // (2^16 is none of f16's: its largest)
      top = (float)(30 - e);
      float corr[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float mx = fmaxf(fmaxf(lg[0][e], lg[1][e]), fmaxf(lg[2][e], lg[3][e]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
        const float mnew = fmaxf(m_run[e], mx - (top - 4.f));
        corr[e] = ex2(m_run[e] - mnew);
        m_run[e] = mnew;
        l_run[e] *= corr[e];
      }
#pragma unroll
      for (int v = 0; v < NP; ++v)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          acc[v][mt][0] *= corr[0]; acc[v][mt][1] *= corr[1];
          acc[v][mt][2] *= corr[0]; acc[v][mt][3] *= corr[1];
        }
      acc_z[0] *= corr[0]; acc_z[1] *= corr[1];
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = ex2(lg[j][e] - m_run[e]);
        l_run[e] += p;
        const __half hv = __float2half_rn(p);
        asm volatile("st.shared.u16 [%0], %1;\n" ::"r"(sP + (2 * t + e) * L::P_STRIDE + (g + 8 * j) * 2),
                     "h"(*reinterpret_cast<const unsigned short*>(&hv)));
      }
    __syncwarp();
    uint32_t p2[4];                                             // tokens (2t, 2t+1) + 8 pr of head g
#pragma unroll
    for (int pr = 0; pr < 4; ++pr) p2[pr] = lds32(sP + g * L::P_STRIDE + 4 * t + 16 * pr);

    // ---- values
    uint32_t zp[4], ps[4][NG];
#pragma unroll
    for (int pr = 0; pr < 4; ++pr) {
      const int tau = 8 * pr + 2 * t;
      __half s0[2 * NG];                                        // groups of token tau, then of tau + 1
      lds_halves(s0, sb + L::VS + tau * NG * 2);
#pragma unroll
      for (int gi = 0; gi < NG; ++gi) {
        const __half2 pair = __halves2half2(s0[gi], s0[NG + gi]);
        ps[pr][gi] = hmul2_u32(p2[pr], *reinterpret_cast<const uint32_t*>(&pair));
      }
      zp[pr] = 0u;                                              // row g < NG: the zero points of group g
      if (g < NG) {
        unsigned short z0, z1;
        asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(z0) : "r"(sb + L::VZ + (tau * NG + g) * 2));
        asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(z1) : "r"(sb + L::VZ + ((tau + 1) * NG + g) * 2));
        zp[pr] = (uint32_t)z0 | (uint32_t)z1 << 16;
      }
    }
    mma_f16_m16n8k16(acc_z, zp[0], 0u, zp[1], 0u, p2[0], p2[1]);
    mma_f16_m16n8k16(acc_z, zp[2], 0u, zp[3], 0u, p2[2], p2[3]);
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
#pragma unroll
      for (int pp = 0; pp < L::PPG; ++pp) {
        const int v = L::SETS > 1 ? gi / L::SETS : gi * L::PPG + pp;
        uint32_t r[4];
        ldmatrix_x4_trans(r[0], r[1], r[2], r[3], sb + L::VC + L::piece(tau_ld, v));
        if (L::SETS > 1 && g / (8 / L::SETS) != gi % L::SETS) r[0] = r[1] = r[2] = r[3] = 0u;   // this lane's unit is the other group's
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint32_t x[4], y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            constexpr uint32_t ones = (1u << BITS) - 1u;
            const int p0 = 2 * mt * BITS, p1 = (2 * mt + 1) * BITS;
            x[i] = (p0 < 8 ? r[i] : r[i] >> 8) & ((ones | ones << 16) << (p0 & 7));
            y[i] = (p1 < 8 ? r[i] : r[i] >> 8) & ((ones | ones << 16) << (p1 & 7));
          }
          mma_f16_m16n8k16(acc[v][mt], x[0], y[0], x[1], y[1], ps[0][gi], ps[1][gi]);
          mma_f16_m16n8k16(acc[v][mt], x[2], y[2], x[3], y[3], ps[2][gi], ps[3][gi]);
        }
      }
    }
    sb_copy = sb;
    sb = sb + L::BYTES == sP ? wsm : sb + L::BYTES;
  }

  // ---- this warp's result: head 2t + e, channel of (piece v, unit g, field)
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    l_run[e] += __shfl_xor_sync(0xffffffffu, l_run[e], 4);
    l_run[e] += __shfl_xor_sync(0xffffffffu, l_run[e], 8);
    l_run[e] += __shfl_xor_sync(0xffffffffu, l_run[e], 16);
  }
  __syncthreads();                                              // the stages are idle
  float* s_acc = reinterpret_cast<float*>(smem);                // [warp][8][D]
  float *s_m = s_acc + DW_WARPS * 8 * D, *s_l = s_m + DW_WARPS * 8, *s_out = s_l + DW_WARPS * 8;
  float2* s_ml = reinterpret_cast<float2*>(s_out + 8 * D);
#pragma unroll
  for (int v = 0; v < NP; ++v) {
    const int grp = (v * L::CH + g * L::U) / GROUP;             // group of this lane's channels: its zero term is with lane (grp, t)
    const float z0 = __shfl_sync(0xffffffffu, acc_z[0], grp * 4 + t), z1 = __shfl_sync(0xffffffffu, acc_z[1], grp * 4 + t);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int f = 2 * mt + half, d = v * L::CH + g * L::U + f;
        const float up = C24 / (float)(1 << ((f * BITS) & 7));
        s_acc[(warp * 8 + 2 * t) * D + d] = fmaf(acc[v][mt][2 * half], up, z0);
        s_acc[(warp * 8 + 2 * t + 1) * D + d] = fmaf(acc[v][mt][2 * half + 1], up, z1);
      }
  }
  if (g == 0)
#pragma unroll
    for (int e = 0; e < 2; ++e) { s_m[warp * 8 + 2 * t + e] = m_run[e]; s_l[warp * 8 + 2 * t + e] = l_run[e]; }
  __syncthreads();
  dw_finish<D, DW_WARPS>(a, bh, G, tok_lo, tok_hi, s_acc, s_m, s_l, s_out, s_ml, lg_out, lstride);
}

// CTAs per (batch, KV head): the cluster size with the shortest schedule.  All CTAs of a launch stream the same number of tiles
// (+-1), `active` clusters of a size fit on the GPU at once, so the launch lasts ceil(heads / active) rounds of (tiles per warp
// + a fixed cost of about two tiles for set-up and exchange).
template <typename K>
cudaError_t launch_dw(K kernel, int warps, int warp_tokens, size_t smem, DwArgs a, int BH, float* ws, int (&active)[64][DW_MAX_CLUSTER + 1],
                      cudaStream_t st) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(warps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  e = clusters_that_fit(kernel, cfg, DW_MAX_CLUSTER, active[dev]);
  if (e != cudaSuccess) return e;
  const int tiles = a.n32 / 32;
  double best = 1e300;
  a.cluster = 1;
  for (int c = 1; c <= DW_MAX_CLUSTER && c <= tiles; ++c) {
    if (active[dev][c] < 1) continue;
    const int per_warp = ((tiles + c - 1) / c * (32 / warp_tokens) + warps - 1) / warps;
    const double cost = (double)((BH + active[dev][c] - 1) / active[dev][c]) * (per_warp + 2);
    if (cost < best) { best = cost; a.cluster = c; }
  }
  const size_t run = (size_t)((tiles + a.cluster - 1) / a.cluster) * 32;
  a.logits = run * (a.Hq / a.Hkv) * sizeof(float) <= DW_LOGIT_BYTES ? nullptr : ws;
  cfg.gridDim = dim3((unsigned)BH * a.cluster);
  attr[0].val.clusterDim.x = a.cluster;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <int BITS, int D, int GROUP>
cudaError_t launch_packed(const DwArgs& a, int BH, float* ws, cudaStream_t st) {
  static int active[64][DW_MAX_CLUSTER + 1] = {};
  return launch_dw(decode_weights_packed_kernel<BITS, D, GROUP>, DW_WARPS, 32, Pk<BITS, D, GROUP>::SMEM_ALL, a, BH, ws, active, st);
}
template <int D>
cudaError_t launch_16(const DwArgs& a, int BH, float* ws, cudaStream_t st) {
  static int active[64][DW_MAX_CLUSTER + 1] = {};
  return launch_dw(decode_weights16_kernel<D>, DW16_WARPS, 16, dw16_smem<D>(), a, BH, ws, active, st);
}
template <int BITS>
cudaError_t launch_bits(const DwArgs& a, int D, int BH, float* ws, cudaStream_t st) {
  if (D == 128) {
    if (a.group == 32) return launch_packed<BITS, 128, 32>(a, BH, ws, st);
    if (a.group == 64) return launch_packed<BITS, 128, 64>(a, BH, ws, st);
    return launch_packed<BITS, 128, 128>(a, BH, ws, st);
  }
  if (a.group == 32) return launch_packed<BITS, 64, 32>(a, BH, ws, st);
  return launch_packed<BITS, 64, 64>(a, BH, ws, st);
}

}  // namespace

size_t decode_weights_workspace(const DecDims& d, int n_cap) {
  return ((size_t)d.Bt * d.Hq * ((n_cap + 31) / 32 * 32) * sizeof(float) + 255) & ~(size_t)255;
}

cudaError_t launch_decode_weights(const DecLayer& ly, const DecDims& d, float* weights, void* ws, cudaStream_t st) {
  DwArgs a{};
  a.ly = ly;
  a.Bt = d.Bt; a.Hq = d.Hq; a.Hkv = d.Hkv; a.group = d.group;
  a.weights = weights;
  a.n32 = (ly.n + 31) / 32 * 32;
  const int BH = d.Bt * d.Hkv;
  float* w = static_cast<float*>(ws);
  switch (d.bits) {
    case 2: return launch_bits<2>(a, d.D, BH, w, st);
    case 4: return launch_bits<4>(a, d.D, BH, w, st);
    case 8: return launch_bits<8>(a, d.D, BH, w, st);
    case 16: return d.D == 128 ? launch_16<128>(a, BH, w, st) : launch_16<64>(a, BH, w, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace qp
