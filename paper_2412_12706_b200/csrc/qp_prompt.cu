// Attention weight the keys of a prompt have received from its queries.
//
// First form: a warp per query row for the normalisers, then a thread per key for the column sums.
#include "qp_common.cuh"

namespace qp {

namespace {

__device__ __forceinline__ float dot_bf16(const uint16_t* a, const uint16_t* b, int D) {
  float s = 0.f;
  for (int d = 0; d < D; d += 2) {
    const uint32_t x = *reinterpret_cast<const uint32_t*>(a + d), y = *reinterpret_cast<const uint32_t*>(b + d);
    s = fmaf(bf16lo(x), bf16lo(y), s);
    s = fmaf(bf16hi(x), bf16hi(y), s);
  }
  return s;
}

// lse[b, h, i] = log2 of the row's sum of 2^(logit), logits in the log2 domain
__global__ void __launch_bounds__(128)
prompt_lse_kernel(const PromptDims d, const uint16_t* __restrict__ Q, const uint16_t* __restrict__ K, float scale_log2,
                  float* __restrict__ lse) {
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= (long long)d.Bt * d.Hq * d.nq) return;
  const int i = (int)(row % d.nq), bq = (int)(row / d.nq), b = bq / d.Hq, h = bq % d.Hq;
  const uint16_t* q = Q + (size_t)row * d.D;
  const uint16_t* k = K + ((size_t)b * d.Hkv + h / (d.Hq / d.Hkv)) * d.L * d.D;
  float m = -INFINITY, s = 0.f;
  for (int j = lane; j <= d.q_start + i; j += 32) {
    const float x = dot_bf16(q, k + (size_t)j * d.D, d.D) * scale_log2, mn = fmaxf(m, x);
    s = s * exp2f(m - mn) + exp2f(x - mn);
    m = mn;
  }
  for (int o = 16; o > 0; o >>= 1) {
    const float mo = __shfl_xor_sync(0xffffffffu, m, o), so = __shfl_xor_sync(0xffffffffu, s, o), mn = fmaxf(m, mo);
    if (mn != -INFINITY) {
      s = s * exp2f(m - mn) + so * exp2f(mo - mn);
      m = mn;
    }
  }
  if (lane == 0) lse[row] = m + log2f(s);
}

__global__ void __launch_bounds__(128)
prompt_columns_kernel(const PromptDims d, const uint16_t* __restrict__ Q, const uint16_t* __restrict__ K, float scale_log2,
                      const float* __restrict__ lse, int accumulate, float* __restrict__ weights) {
  const int bh = blockIdx.y, b = bh / d.Hkv, hk = bh % d.Hkv, G = d.Hq / d.Hkv, j = blockIdx.x * 128 + threadIdx.x;
  if (j >= d.L) return;
  float acc = 0.f;
  if (j < d.q_start + d.nq) {
    const uint16_t* k = K + ((size_t)bh * d.L + j) * d.D;
    for (int g = 0; g < G; ++g) {
      const size_t row0 = ((size_t)b * d.Hq + hk * G + g) * d.nq;
      float part = 0.f;
      for (int i = max(0, j - d.q_start); i < d.nq; ++i)
        part += exp2f(dot_bf16(Q + (row0 + i) * d.D, k, d.D) * scale_log2 - lse[row0 + i]);
      acc += part;
    }
  }
  float* w = weights + (size_t)bh * d.L + j;
  if (!accumulate) *w = acc;
  else if (j < d.q_start + d.nq) *w += acc;
}

}  // namespace

size_t prompt_workspace(const PromptDims& d) { return (((size_t)d.Bt * d.Hq * d.nq * sizeof(float) + 255) & ~(size_t)255) + 256; }

cudaError_t launch_prompt_weights(const void* Q, const void* K, const PromptDims& d, int accumulate, float* weights, void* ws,
                                  cudaStream_t st) {
  float* lse = static_cast<float*>(ws);
  const uint16_t *q = static_cast<const uint16_t*>(Q), *k = static_cast<const uint16_t*>(K);
  const float scale_log2 = (float)(1.4426950408889634 / sqrt((double)d.D));
  cudaError_t e = cudaMemsetAsync(static_cast<char*>(ws) + prompt_workspace(d) - 256, 0, 4, st);
  if (e != cudaSuccess) return e;
  const long long rows = (long long)d.Bt * d.Hq * d.nq;
  prompt_lse_kernel<<<(unsigned)((rows + 3) / 4), 128, 0, st>>>(d, q, k, scale_log2, lse);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  prompt_columns_kernel<<<dim3((d.L + 127) / 128, d.Bt * d.Hkv), 128, 0, st>>>(d, q, k, scale_log2, lse, accumulate, weights);
  return cudaGetLastError();
}

}  // namespace qp
