// Attention of a tree of drafted tokens over a packed cache, its tail and the drafts themselves.
//
// First form: one block per (draft, batch, KV head), SIMT arithmetic, 128 tokens at a time.
#include "qp_common.cuh"

namespace qp {

namespace {

__device__ __forceinline__ float code_value(const void* codes, const __half* scale, const __half* zero, size_t grp, int e, int g,
                                            int bits) {
  const int per = 32 / bits;
  const uint32_t word = static_cast<const uint32_t*>(codes)[grp * (g * bits / 32) + e / per];
  const float c = (float)((word >> ((e % per) * bits)) & ((1u << bits) - 1u));
  return fmaf(c, __half2float(scale[grp]), __half2float(zero[grp]));
}

__global__ void __launch_bounds__(128)
tree_simple_kernel(const TreeArgs a) {
  __shared__ float s_q[8][128], s_p[8][128], s_red[4];
  const int t = blockIdx.x, bh = blockIdx.y, b = bh / a.Hkv, hk = bh % a.Hkv, tid = threadIdx.x, D = a.D, G = a.Hq / a.Hkv, g = a.group;
  const uint16_t* q = static_cast<const uint16_t*>(a.q) + (((size_t)b * a.T + t) * a.Hq + hk * G) * D;
  const float scale_log2 = 1.4426950408889634f * rsqrtf((float)D);
  for (int i = tid; i < G * D; i += 128) s_q[i / D][i % D] = bf16_bits_to_f32(q[i]) * scale_log2;
  __syncthreads();
  const unsigned long long mask = a.mask[(size_t)b * a.T + t];
  const int total = a.n + a.n_tail + a.T;
  const uint16_t *kt = static_cast<const uint16_t*>(a.k_tail), *vt = static_cast<const uint16_t*>(a.v_tail);
  const uint16_t *kd = static_cast<const uint16_t*>(a.k_draft), *vd = static_cast<const uint16_t*>(a.v_draft);
  auto element = [&](bool key, int x, int d) {
    if (x < a.n) {
      const size_t row = (size_t)bh * a.ns + x;
      if (a.bits == 16) return bf16_bits_to_f32(static_cast<const uint16_t*>(key ? a.kc : a.vc)[row * D + d]);
      if (key && a.k_axis == 0)
        return code_value(a.kc, a.ks, a.kz, ((size_t)bh * (a.ns / g) + x / g) * D + d, x % g, g, a.bits);
      const size_t grp = row * (D / g) + d / g;
      return key ? code_value(a.kc, a.ks, a.kz, grp, d % g, g, a.bits) : code_value(a.vc, a.vs, a.vz, grp, d % g, g, a.bits);
    }
    if (x < a.n + a.n_tail) return bf16_bits_to_f32((key ? kt : vt)[((size_t)bh * g + (x - a.n)) * D + d]);
    return bf16_bits_to_f32((key ? kd : vd)[(((size_t)b * a.T + (x - a.n - a.n_tail)) * a.Hkv + hk) * D + d]);
  };
  float m[8], l[8], o[8];
  for (int h = 0; h < G; ++h) { m[h] = -INFINITY; l[h] = 0.f; o[h] = 0.f; }
  for (int x0 = 0; x0 < total; x0 += 128) {
    const int x = x0 + tid, e = x - a.n - a.n_tail;
    const bool sees = x < total && (e < 0 || ((mask >> e) & 1ull));
    float acc[8] = {};
    if (sees)
      for (int d = 0; d < D; ++d) {
        const float k = element(true, x, d);
        for (int h = 0; h < G; ++h) acc[h] = fmaf(s_q[h][d], k, acc[h]);
      }
    for (int h = 0; h < G; ++h) {
      const float v = sees ? acc[h] : -INFINITY;
      float mx = v;
      for (int s = 16; s > 0; s >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
      __syncthreads();
      if ((tid & 31) == 0) s_red[tid >> 5] = mx;
      __syncthreads();
      const float mn = fmaxf(m[h], fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])));
      const float p = sees ? exp2f(v - mn) : 0.f, corr = mn == -INFINITY ? 1.f : exp2f(m[h] - mn);
      s_p[h][tid] = p;
      __syncthreads();
      m[h] = mn;
      float sum = 0.f;
      for (int i = 0; i < 128; ++i) sum += s_p[h][i];
      l[h] = l[h] * corr + sum;
      o[h] *= corr;
    }
    if (tid < D)
      for (int i = 0; i < min(128, total - x0); ++i) {
        const int xi = x0 + i, ei = xi - a.n - a.n_tail;
        if (ei >= 0 && !((mask >> ei) & 1ull)) continue;
        const float v = element(false, xi, tid);
        for (int h = 0; h < G; ++h) o[h] = fmaf(s_p[h][i], v, o[h]);
      }
    __syncthreads();
  }
  if (tid < D)
    for (int h = 0; h < G; ++h)
      static_cast<bf16*>(a.out)[(((size_t)b * a.T + t) * a.Hq + hk * G + h) * D + tid] = __float2bfloat16_rn(o[h] / l[h]);
}

}  // namespace

size_t tree_workspace(const TreeArgs&) { return 256; }

cudaError_t launch_tree(const TreeArgs& a, void* ws, cudaStream_t st) {
  const cudaError_t e = cudaMemsetAsync(static_cast<char*>(ws) + tree_workspace(a) - 256, 0, 4, st);
  if (e != cudaSuccess) return e;
  tree_simple_kernel<<<dim3(a.T, a.Bt * a.Hkv), 128, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace qp
