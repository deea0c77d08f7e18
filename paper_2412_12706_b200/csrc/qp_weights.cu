// The two forms of the eviction by accumulated attention weight: the state of a cache after a prompt's selection, and the
// replacement of one token per step.
#include "qp_common.cuh"

namespace qp {

namespace {

// state of a cache filled with the kept tokens: their weights and positions, zero behind them
__global__ void __launch_bounds__(256)
kept_state_kernel(const float* __restrict__ weights, const int32_t* __restrict__ kept, int L, int n, int cap,
                  float* __restrict__ kw, int32_t* __restrict__ kp) {
  const int bh = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  if (i >= cap) return;
  const int src = i < n ? kept[(size_t)bh * n + i] : 0;
  if (kw) kw[(size_t)bh * cap + i] = i < n ? weights[(size_t)bh * L + src] : 0.f;
  if (kp) kp[(size_t)bh * cap + i] = src;
}

// monotone map float -> uint32 (larger float = larger integer); -0 as +0
__device__ __forceinline__ uint32_t order_image(float f) {
  const uint32_t u = __float_as_uint(f + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ void quantize_row_group(const uint16_t* x, int g, int bits, uint32_t* words, __half* scale, __half* zero) {
  const int qmax = (1 << bits) - 1, per = 32 / bits;
  float mn = INFINITY, mx = -INFINITY;
  for (int e = 0; e < g; ++e) {
    const float v = bf16_bits_to_f32(x[e]);
    mn = fminf(mn, v);
    mx = fmaxf(mx, v);
  }
  const __half z16 = __float2half_rd(mn);
  const float z = __half2float(z16);
  const __half s16 = __float2half_ru(__fmul_rn(__fsub_rn(mx, z), 1.0f / (float)qmax));   // product with the rounded reciprocal
  const float s = __half2float(s16);
  for (int w = 0; w < g / per; ++w) {
    uint32_t word = 0;
    for (int i = 0; i < per; ++i) {
      const float c = s > 0.f ? rintf(__fdiv_rn(__fsub_rn(bf16_bits_to_f32(x[w * per + i]), z), s)) : 0.f;
      word |= (uint32_t)fminf(fmaxf(c, 0.f), (float)qmax) << (i * bits);
    }
    words[w] = word;
  }
  *scale = s16;
  *zero = z16;
}

// one block per (batch, KV head): the slot, then the row
__global__ void __launch_bounds__(256)
evict_kernel(const EvictArgs a) {
  __shared__ unsigned long long s_light[8], s_old[8];
  const int bh = blockIdx.x, tid = threadIdx.x;
  float* w = a.weights + (size_t)bh * a.ns;
  int32_t* pos = a.pos + (size_t)bh * a.ns;
  int slot = a.slot;
  if (slot < 0) {
    unsigned long long light = ~0ull, oldest = ~0ull;
    for (int t = tid; t < a.n; t += 256) {
      const int p = pos[t];
      const unsigned long long o = ((unsigned long long)((uint32_t)p ^ 0x80000000u) << 32) | (unsigned)t;
      oldest = o < oldest ? o : oldest;
      if ((long long)p <= a.limit) {
        const unsigned long long k = ((unsigned long long)order_image(w[t]) << 32) | (unsigned)t;
        light = k < light ? k : light;
      }
    }
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long x = __shfl_xor_sync(0xffffffffu, light, o), y = __shfl_xor_sync(0xffffffffu, oldest, o);
      light = x < light ? x : light;
      oldest = y < oldest ? y : oldest;
    }
    if ((tid & 31) == 0) { s_light[tid >> 5] = light; s_old[tid >> 5] = oldest; }
    __syncthreads();
    light = s_light[0]; oldest = s_old[0];
    for (int i = 1; i < 8; ++i) {
      light = s_light[i] < light ? s_light[i] : light;
      oldest = s_old[i] < oldest ? s_old[i] : oldest;
    }
    slot = (int)(uint32_t)(light != ~0ull ? light : oldest);
  }
  const int D = a.D, g = a.g;
  const size_t row = (size_t)bh * a.ns + slot;
  const uint16_t *k = a.k_new + (size_t)bh * D, *v = a.v_new + (size_t)bh * D;
  if (a.bits == 16) {
    for (int d = tid; d < D; d += 256) {
      static_cast<uint16_t*>(a.kc)[row * D + d] = k[d];
      static_cast<uint16_t*>(a.vc)[row * D + d] = v[d];
    }
  } else if (tid < 2 * (D / g)) {
    const int grp = tid >> 1, wpg = g * a.bits / 32;
    const size_t gi = row * (D / g) + grp;
    if (tid & 1) quantize_row_group(v + grp * g, g, a.bits, static_cast<uint32_t*>(a.vc) + gi * wpg, a.vs + gi, a.vz + gi);
    else quantize_row_group(k + grp * g, g, a.bits, static_cast<uint32_t*>(a.kc) + gi * wpg, a.ks + gi, a.kz + gi);
  }
  if (tid == 0) {
    w[slot] = 0.f;
    pos[slot] = a.new_pos;
    if (a.slots) a.slots[bh] = slot;
  }
}

}  // namespace

cudaError_t launch_kept_state(const float* weights, const int32_t* kept, int BH, int L, int n, int cap, float* kw, int32_t* kp,
                              cudaStream_t st) {
  kept_state_kernel<<<dim3((cap + 255) / 256, BH), 256, 0, st>>>(weights, kept, L, n, cap, kw, kp);
  return cudaGetLastError();
}

cudaError_t launch_evict(const EvictArgs& a, int BH, cudaStream_t st) {
  evict_kernel<<<BH, 256, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace qp
