// Eviction by accumulated attention weight, one token per step (the prompt's form is a selection: qp_topk.cu).
#include "qp_common.cuh"

namespace qp {

namespace {

// One block per (batch, KV head).  The call is a chain of latencies (a few hundred KB in all): the row is fetched and quantized
// while the search's loads are on their way, every thread has EV_PER weights and positions in flight, and the two minima the
// rule may need (lightest of the old, oldest of all) are taken together as 64-bit keys (order image, slot), which makes equal
// values go to the lower slot.  Measured in a replayed graph: 512 slots x 8 heads at 16 bit 2.9 us, 8192 x 64 heads at 4 bit 4.7.
constexpr int EV_THREADS = 1024, EV_PER = 8;

// code of one element, RN((x - z) / s) clamped
__device__ __forceinline__ uint32_t code_of(float x, float z, float s, int qmax) {
  const float c = s > 0.f ? rintf(__fdiv_rn(__fsub_rn(x, z), s)) : 0.f;
  return (uint32_t)fminf(fmaxf(c, 0.f), (float)qmax);
}

__global__ void __launch_bounds__(EV_THREADS)
evict_kernel(const __grid_constant__ EvictArgs a) {
  __shared__ unsigned long long s_light[EV_THREADS / 32], s_old[EV_THREADS / 32];
  __shared__ int s_slot;
  const int bh = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int D = a.D, g = a.g, ngv = D / g;
  chain_enter();
  float* w = a.weights + (size_t)bh * a.ns;
  int32_t* pos = a.pos + (size_t)bh * a.ns;

  // the row: packed caches, a warp per group (keys, then values), up to four elements a lane; 16 bit, 16-byte pieces
  const bool quant = a.bits < 16 && warp < 2 * ngv, key = warp < ngv;
  const int grp = key ? warp : warp - ngv, per_lane = g / 32;
  const uint16_t* src = (key ? a.k_new : a.v_new) + (size_t)bh * D + grp * g;
  float x[4];
  uint4 piece;
  if (quant) {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = k < per_lane ? bf16_bits_to_f32(src[lane * per_lane + k]) : 0.f;
  } else if (a.bits == 16 && tid < D / 4) {
    piece = *reinterpret_cast<const uint4*>((tid < D / 8 ? a.k_new : a.v_new) + (size_t)bh * D + (tid % (D / 8)) * 8);
  }

  int slot = a.slot;
  unsigned long long light = ~0ull, oldest = ~0ull;
  if (slot < 0)
    for (int t0 = tid; t0 < a.n; t0 += EV_PER * EV_THREADS) {
      int32_t p[EV_PER];
      float v[EV_PER];
#pragma unroll
      for (int k = 0; k < EV_PER; ++k) {
        const int t = min(t0 + k * EV_THREADS, a.n - 1);        // past the end: the last one again
        p[k] = pos[t];
        v[k] = w[t];
      }
#pragma unroll
      for (int k = 0; k < EV_PER; ++k) {
        const unsigned t = (unsigned)min(t0 + k * EV_THREADS, a.n - 1);
        const unsigned long long o = ((unsigned long long)((uint32_t)p[k] ^ 0x80000000u) << 32) | t;
        const unsigned long long l = (long long)p[k] <= a.limit ? ((unsigned long long)order_key(v[k]) << 32) | t : ~0ull;
        oldest = o < oldest ? o : oldest;
        light = l < light ? l : light;
      }
    }

  // quantization of this warp's group (its loads came first)
  uint32_t word = 0;
  __half s16, z16;
  if (quant) {
    const int qmax = (1 << a.bits) - 1, bits = a.bits;
    float mn = x[0], mx = x[0];
#pragma unroll
    for (int k = 1; k < 4; ++k)
      if (k < per_lane) { mn = fminf(mn, x[k]); mx = fmaxf(mx, x[k]); }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    }
    z16 = __float2half_rd(mn);
    const float z = __half2float(z16);
    // The product with the rounded reciprocal, where the prompt's quantizer takes the rounded quotient: what tensor code stores that
    // divides a row on the GPU by the number 2^B - 1, so that such code and this call agree bit for bit.  RN(1/3), RN(1/15) and
    // RN(1/255) lie above the reciprocals: the scale is the quotient's or one fp16 step more, never less, and nothing clips.
    s16 = __float2half_ru(__fmul_rn(__fsub_rn(mx, z), 1.0f / (float)qmax));
    const float s = __half2float(s16);
    // this lane's elements fill per_lane * bits bits of a word; the lanes of a word put theirs together
    const int lanes = 32 / (per_lane * bits), sub = lanes > 1 ? lane % lanes : 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < per_lane) word |= code_of(x[k], z, s, qmax) << (((sub * per_lane + k) * bits) & 31);
    for (int o = 1; o < lanes; o <<= 1) word |= __shfl_xor_sync(0xffffffffu, word, o);
  }

  if (slot < 0) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long l = __shfl_xor_sync(0xffffffffu, light, o), y = __shfl_xor_sync(0xffffffffu, oldest, o);
      light = l < light ? l : light;
      oldest = y < oldest ? y : oldest;
    }
    if (lane == 0) { s_light[warp] = light; s_old[warp] = oldest; }
    __syncthreads();
    if (warp == 0) {
      light = s_light[lane];
      oldest = s_old[lane];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long l = __shfl_xor_sync(0xffffffffu, light, o), y = __shfl_xor_sync(0xffffffffu, oldest, o);
        light = l < light ? l : light;
        oldest = y < oldest ? y : oldest;
      }
      if (lane == 0) s_slot = (int)(uint32_t)(light != ~0ull ? light : oldest);
    }
    __syncthreads();
    slot = s_slot;
  }

  const size_t row = (size_t)bh * a.ns + slot;
  if (quant) {
    const size_t gi = row * ngv + grp;
    const int lanes = 32 / (per_lane * a.bits);
    uint32_t* words = static_cast<uint32_t*>(key ? a.kc : a.vc) + gi * (g * a.bits / 32);
    if (lane % lanes == 0) words[lane / lanes] = word;
    if (lane == 0) {
      (key ? a.ks : a.vs)[gi] = s16;
      (key ? a.kz : a.vz)[gi] = z16;
    }
  } else if (a.bits == 16 && tid < D / 4) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(tid < D / 8 ? a.kc : a.vc) + row * D + (tid % (D / 8)) * 8) = piece;
  }
  if (tid == EV_THREADS - 1) {
    w[slot] = 0.f;
    pos[slot] = a.new_pos;
    if (a.slots) a.slots[bh] = slot;
  }
}

}  // namespace

cudaError_t launch_evict(const EvictArgs& a, int BH, cudaStream_t st) {
  return launch_chained(evict_kernel, dim3(BH), dim3(EV_THREADS), 0, st, a);
}

}  // namespace qp
