// Position rotation and the paged cache in 8 bits: what their kernels share, and their launchers.
#pragma once

#include <cuda.h>

#include "qp_checked.cuh"
#include "qp_common.cuh"

namespace qp {

// The arrays of a step on the device, and what the host says of them.
struct StepView {
  const int32_t *start, *len, *pages;
  int n_seqs, n_tokens, max_new, max_pages, page, n_pages;
};
// Sequence b of a step: rows row0 .. row0 + n - 1 of the step's arrays stand at positions len .. len + n - 1.  Numbers that do not
// belong together (rows outside the arrays, more tokens than the host said, more than the page table's row holds) give n = 0: the
// sequence is left out, and nothing is addressed by them.  (The range-checked build records them, too.)
struct Seq {
  int row0, n, len;
};
__device__ __forceinline__ Seq seq_of(const StepView& s, int b) {
  const int r0 = __ldg(s.start + b), r1 = __ldg(s.start + b + 1), len = __ldg(s.len + b);
  const bool rows = r0 >= 0 && r1 >= r0 && r1 <= s.n_tokens && r1 - r0 <= s.max_new;
  const bool ok = rows && len >= 0 && (long long)len + (r1 - r0) <= (long long)s.max_pages * s.page;
#ifdef QP_CHECKED
  if (!rows) {
    if (QP_IN_RANGE(r0, s.n_tokens + 1LL, QP_SITE_STEP_START)) QP_IN_RANGE((long long)r1 - r0, min(s.max_new, s.n_tokens - r0) + 1LL, QP_SITE_STEP_START);
  } else if (r1 > r0) {
    QP_IN_RANGE(len, (long long)s.max_pages * s.page - (r1 - r0) + 1, QP_SITE_STEP_LEN);
  }
#endif
  return Seq{r0, ok ? r1 - r0 : 0, len};
}
// page i of sequence b; one that is outside the pool becomes -1
__device__ __forceinline__ int page_of(const StepView& s, int b, int i) {
  const int p = __ldg(s.pages + (size_t)b * s.max_pages + i);
  const bool ok = (unsigned)p < (unsigned)s.n_pages;
#ifdef QP_CHECKED
  if (!ok) QP_IN_RANGE(p, s.n_pages, QP_SITE_STEP_PAGE);
#endif
  return ok ? p : -1;
}

struct RotaryArgs {
  const uint16_t* x;
  uint16_t* out;
  long long xs[3], os[3], ps;     // strides in elements: batch, head, token; positions: batch
  const int32_t* pos;
  int Bt, H, L, D, transpose;
};
cudaError_t launch_rotary(const RotaryArgs& a, const qp_rope& rope, cudaStream_t st);

struct AppendArgs {
  StepView s;
  const uint16_t *k, *v, *q;      // new rows [n_tokens][heads][D]; q null: none to rotate
  uint16_t* q_out;
  long long ks, vs, qs;           // elements from a token's row to the next
  const int32_t* pos;             // null: the positions in the sequences
  uint8_t *kc, *vc;               // [n_pages][Hkv][page][D]
  uint16_t *k_scale, *v_scale;    // bf16 [n_pages][Hkv]
  uint16_t *k_tail, *v_tail;      // bf16 [n_seqs][Hkv][page][D]
  int Hq, Hkv, D, format;
};
cudaError_t launch_paged_append(const AppendArgs& a, const qp_rope* rope, cudaStream_t st);

struct PagedAttnArgs {
  StepView s;
  const uint16_t* q;
  long long qs;
  uint16_t* out;                  // [n_tokens][Hq][D]
  const uint8_t *kc, *vc;
  const uint16_t *k_scale, *v_scale;
  const uint16_t *k_tail, *v_tail;
  int Hq, Hkv, D, format;
};
// whether the work of a call can be numbered in 31 bits, with sequences as long as the page table allows
bool paged_attn_fits(int n_seqs, int n_tokens, int max_new, int Hq, int Hkv, long long most_len);
size_t paged_attn_workspace(int n_seqs, int n_tokens, int max_new, int Hq, int Hkv, int D);
cudaError_t launch_paged_attn(const PagedAttnArgs& a, void* ws, cudaStream_t st);
// the form for many query rows per KV head; mk, mv: the codes as rows of D bytes, boxes of 32 of them
bool paged_chunk_fits(int n_seqs, int n_tokens, int Hq, int Hkv, long long most_len);
size_t paged_chunk_workspace(int n_seqs, int n_tokens, int Hq, int Hkv, int D);
cudaError_t launch_paged_chunk(const PagedAttnArgs& a, void* ws, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t st);

}  // namespace qp
