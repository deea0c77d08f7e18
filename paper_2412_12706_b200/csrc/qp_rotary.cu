// Rotation by position (qp_rotary) and the appends to a paged cache in 8 bits (qp_paged_append).
//
// A pair (u, v) of channels turns by the angle a = pos * w:  u' = m (u cos a - v sin a),  v' = m (v cos a + u sin a).  What counts of
// pos * w is its fraction of a full turn, so w is held as w / 2 pi in units of 2^-64 and the product taken in 64-bit integers, whose
// overflow drops the whole turns: at any 31-bit position it is off by 2^-34 of a turn, from the rounding of w.  The cosine and sine are
// taken of its upper 32 bits, rounded to multiples of 2^-25 of a turn: off by 2^-26 of a turn, 1e-7 radians, where a 32-bit float angle
// is off by 0.06 at a million.
#include <algorithm>
#include <cfloat>

#include "qp_paged.cuh"

namespace qp {

namespace {

constexpr int THREADS = 128;
constexpr int ROT_TOKENS = 32;                                  // most tokens of a rotation's block

// how the channels pair up: neighbours; i with i + rot/2 where rot/2 is a whole number of 16-byte vectors; the same where it is not
enum : int { PAIR_NEXT = 0, PAIR_HALF = 1, PAIR_ODD = 2 };
inline int pairing(const qp_rope& r) { return r.interleaved ? PAIR_NEXT : r.rot_dim % 16 == 0 ? PAIR_HALF : PAIR_ODD; }

// Cosine and sine, times m, of pair `turn` at position pos.  The upper half of the product is the fraction of a turn in units of 2^-32:
// two bits of quadrant, and the rest as y in [-1/2, 1/2] quarter turns, rounded to multiples of 2^-23.  sin(y pi/2) / y and cos(y pi/2)
// are polynomials in y^2, degree 3 and 4, fitted here by linear programming on [0, 1/4] for the least largest error; with coefficients
// of 32 bits they are off by 5.3e-8 and 3.5e-9.  In 32-bit arithmetic both results are within 9e-8, the rounding of y included within
// 2^-22.  (sincospif and a conversion to float in its place, with the rows asked for after the table: 8192 tokens x 32 heads x 128 in
// 28.4 us, against 25.4 then.)
__device__ __forceinline__ float2 cos_sin(uint64_t turn, int pos, float m) {
  const uint32_t frac = (uint32_t)((turn * (uint64_t)(int64_t)pos) >> 32) + 0x20000000u;
  const uint32_t quarter = frac >> 30;
  const float y = __uint_as_float(0x3f800000u + (((frac & 0x3fffffffu) + 64u) >> 7)) - 1.5f, z = y * y;
  float s = fmaf(-0x1.2d9c3p-8f, z, 0x1.465ecap-4f), c = fmaf(0x1.d6b52cp-11f, z, -0x1.55ba3ep-6f);
  s = fmaf(s, z, -0x1.4abbbap-1f);
  c = fmaf(c, z, 0x1.03c1c4p-2f);
  s = fmaf(s, z, 0x1.921fb6p+0f);
  c = fmaf(c, z, -0x1.3bd3ccp+0f);
  s *= y * m;
  c = fmaf(c, z, 1.f) * m;
  // a quarter turn on: (c, s) -> (-s, c)
  const float a = quarter & 1u ? s : c, b = quarter & 1u ? c : s;
  return make_float2(__uint_as_float(__float_as_uint(a) ^ ((quarter + 1u) & 2u) << 30), __uint_as_float(__float_as_uint(b) ^ (quarter & 2u) << 30));
}

// A unit is 16 channels of a row: two vectors of 8, numbers c0 and c1, such that pairs of PAIR_NEXT and PAIR_HALF lie inside it.
__device__ __forceinline__ void unit_vectors(int mode, int rot, int u, int& c0, int& c1) {
  const int half = rot >> 4;                                    // vectors in half of the rotated part
  const bool across = mode == PAIR_HALF && u < half;
  c0 = across ? u : 2 * u;
  c1 = across ? u + half : 2 * u + 1;
}
// x c + y s, rounded as written here wherever it is: what a page holds must not depend on the kernel that a token came in with
__device__ __forceinline__ float turned(float x, float c, float y, float s) { return fmaf(x, c, __fmul_rn(y, s)); }
// Rotates a unit whose vectors are a and b.  cs2(i): cosines and sines of pairs i and i + 1, i even.  row: the row itself, which PAIR_ODD reads again.
template <int MODE, typename CS>
__device__ __forceinline__ void rotate_unit(uint4& a, uint4& b, int u, int rot, const uint16_t* row, CS cs2) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (MODE == PAIR_NEXT) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const int p = 8 * u + i;
      if (2 * p < rot) {
        const float4 t = cs2(p);
        const float x = bf16lo(w[i]), y = bf16hi(w[i]), z = bf16lo(w[i + 1]), v = bf16hi(w[i + 1]);
        w[i] = pack_bf16x2(turned(x, t.x, -y, t.y), turned(y, t.x, x, t.y));
        if (2 * p + 2 < rot) w[i + 1] = pack_bf16x2(turned(z, t.z, -v, t.w), turned(v, t.z, z, t.w));
      }
    }
  } else if (MODE == PAIR_HALF) {
    if (16 * u < rot) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 t = cs2(8 * u + 2 * i);
        const float x0 = bf16lo(w[i]), x1 = bf16hi(w[i]), y0 = bf16lo(w[4 + i]), y1 = bf16hi(w[4 + i]);
        w[i] = pack_bf16x2(turned(x0, t.x, -y0, t.y), turned(x1, t.z, -y1, t.w));
        w[4 + i] = pack_bf16x2(turned(y0, t.x, x0, t.y), turned(y1, t.z, x1, t.w));
      }
    }
  } else {
    const int half = rot >> 1;
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
      float o[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int d = 16 * u + 2 * i + j;
        const float x = bf16_bits_to_f32(row[d]);
        o[j] = x;
        if (d < rot) {
          const int p = d < half ? d : d - half;
          const float4 both = cs2(p & ~1);
          const float2 t = p & 1 ? make_float2(both.z, both.w) : make_float2(both.x, both.y);
          const float y = bf16_bits_to_f32(row[d < half ? d + half : d - half]);
          o[j] = turned(x, t.x, d < half ? -y : y, t.y);
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k == i) w[k] = pack_bf16x2(o[0], o[1]);
    }
  }
  a = make_uint4(w[0], w[1], w[2], w[3]);
  b = make_uint4(w[4], w[5], w[6], w[7]);
}

// Where pair p stands in its token's part of the table: the first two pairs of every unit, then the next two of every unit, ..., so that
// the lanes of a row read 16 bytes each, one behind the other (in order, four of them meet in the same banks: 8192 tokens x 32 heads x 128
// 25.3 us, against 19.4)
__device__ __forceinline__ int table_place(int p, int pitch) { return ((p & 6) >> 1) * (pitch >> 2) + (p >> 3) * 2 + (p & 1); }

// ---- rotation alone, and of a step's queries.  HBM-bound: 4 bytes a number.  A block takes up to 32 tokens of all heads, so that
// the cosines and sines are computed once a token and read from shared memory by every head.  8192 tokens x 32 heads x 128: 22.7 us over
// changing inputs, 5.9 TB/s (19.4 where a graph writes one output over and over, which stays in L2: the figures compared below).
// Half layout with rot_dim no multiple of 16 (PAIR_ODD) reads its rows again by scalars: 88.8 us with 44 channels.
// The rows are asked for before the table is made (fill, which ends with the block's barrier), so that the two wait together.
// n < 2^16 / H tokens; inv_h = ceil(2^32 / H), or 0 for one head.  pitch: pairs of a token in the table.
template <int MODE, int ROT_UNITS, typename OK, typename FILL>
__device__ __forceinline__ void rotate_tokens(const uint16_t* x, long long xh, long long xl, uint16_t* out, long long oh, long long ol,
                                              int n, int H, uint32_t inv_h, int lgu, int rot, const float2* table, int pitch, OK ok, FILL fill) {
  const int units = (n * H) << lgu;                             // 2^lgu units a row
  for (int base = 0; base < units; base += THREADS * ROT_UNITS) {
    uint4 a[ROT_UNITS], b[ROT_UNITS];
    const uint16_t* src[ROT_UNITS];
    uint16_t* dst[ROT_UNITS];
    int tok[ROT_UNITS];
    const int u = threadIdx.x & ((1 << lgu) - 1);
    int c0, c1;
    unit_vectors(MODE, rot, u, c0, c1);
#pragma unroll
    for (int k = 0; k < ROT_UNITS; ++k) {
      const int i = base + k * THREADS + threadIdx.x, r = i >> lgu, t = inv_h ? __umulhi((uint32_t)r, inv_h) : r, h = r - t * H;
      tok[k] = t;
      src[k] = x + h * xh + t * xl;
      dst[k] = out + h * oh + t * ol;
      if (i < units) {
        a[k] = *reinterpret_cast<const uint4*>(src[k] + 8 * c0);
        b[k] = *reinterpret_cast<const uint4*>(src[k] + 8 * c1);
      }
    }
    if (base == 0) fill();
#pragma unroll
    for (int k = 0; k < ROT_UNITS; ++k)
      if (base + k * THREADS + (int)threadIdx.x < units)
        rotate_unit<MODE>(a[k], b[k], u, rot, src[k], [&](int p) { return *reinterpret_cast<const float4*>(table + tok[k] * pitch + table_place(p, pitch)); });
    if (MODE == PAIR_ODD) __syncwarp();                         // in place: a row's units are one warp's, all read before one writes
#pragma unroll
    for (int k = 0; k < ROT_UNITS; ++k)
      if (base + k * THREADS + (int)threadIdx.x < units && ok(tok[k])) {
        *reinterpret_cast<uint4*>(dst[k] + 8 * c0) = a[k];
        *reinterpret_cast<uint4*>(dst[k] + 8 * c1) = b[k];
      }
  }
}
__host__ __device__ inline int table_pitch(int rot) { return ((rot >> 1) + 7) & ~7; }
uint32_t inverse_of(int H) { return H == 1 ? 0u : (uint32_t)(((1ull << 32) + H - 1) / H); }
// Units a thread has in flight: four where that still leaves every SM its eight blocks (8192 tokens x 32 heads x 128: 19.4 us, against
// 24.7 with one), else one, so that short calls spread over the SMs (3 x 5001 tokens x 8 heads x 64: 6.2 us against 9.5).
int units_a_thread(long long rows, int D) { return rows * (D / 16) >= 148LL * 8 * THREADS * 4 ? 4 : 1; }
// tokens of a block of THREADS * `units` units, but no more than the table holds
int tokens_a_block(int H, int D, int units) { return std::max(1, std::min(ROT_TOKENS, THREADS * units / (H * (D / 16)))); }

template <int MODE, int ROT_UNITS>
__global__ void __launch_bounds__(THREADS)
rotary_kernel(const __grid_constant__ RotaryArgs a, const __grid_constant__ qp_rope rope, int tokens, uint32_t inv_h) {
  __shared__ __align__(16) float2 table[ROT_TOKENS * 64];
  chain_enter();
  const int t0 = blockIdx.x * tokens, n = min(tokens, a.L - t0), half = rope.rot_dim >> 1, pitch = table_pitch(rope.rot_dim);
  for (int b = blockIdx.y; b < a.Bt; b += gridDim.y) {
    auto fill = [&]() {
      for (int i = threadIdx.x; i < n * pitch; i += THREADS) {
        const int t = i / pitch, p = i - t * pitch;
        if (p >= half) continue;
        float2 cs = cos_sin(rope.turn[p], __ldg(a.pos + b * a.ps + t0 + t), rope.factor);
        if (a.transpose) cs.y = -cs.y;
        table[t * pitch + table_place(p, pitch)] = cs;
      }
      __syncthreads();
    };
    rotate_tokens<MODE, ROT_UNITS>(a.x + b * a.xs[0] + t0 * a.xs[2], a.xs[1], a.xs[2], a.out + b * a.os[0] + t0 * a.os[2], a.os[1], a.os[2], n,
                        a.H, inv_h, a.D == 128 ? 3 : 2, rope.rot_dim, table, pitch, [](int) { return true; }, fill);
    __syncthreads();
  }
}

// ---- appends

// largest b < n for which f(start[b]) is not above x, 0 if there is none
template <typename F>
__device__ __forceinline__ int last_at_most(const int32_t* start, int n, int x, F f) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (f(__ldg(start + mid)) <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// codes of 8 numbers
__device__ __forceinline__ uint2 codes8(const uint4& v, float inv, bool e4m3) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t o[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float x0 = __fmul_rn(bf16lo(w[2 * i]), inv), x1 = __fmul_rn(bf16hi(w[2 * i]), inv);
    const float x2 = __fmul_rn(bf16lo(w[2 * i + 1]), inv), x3 = __fmul_rn(bf16hi(w[2 * i + 1]), inv);
    if (e4m3) {
      uint16_t lo, hi;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(lo) : "f"(x1), "f"(x0));
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(hi) : "f"(x3), "f"(x2));
      o[i] = lo | (uint32_t)hi << 16;
    } else {
      auto code = [](float x) { return (uint32_t)__float2int_rn(fminf(fmaxf(x, -127.f), 127.f)) & 0xffu; };
      o[i] = code(x0) | code(x1) << 8 | code(x2) << 16 | code(x3) << 24;
    }
  }
  return make_uint2(o[0], o[1]);
}
__device__ __forceinline__ uint32_t abs_max2(uint32_t m, const uint4& v) {
  m = __vmaxu2(m, v.x & 0x7fff7fffu);
  m = __vmaxu2(m, v.y & 0x7fff7fffu);
  m = __vmaxu2(m, v.z & 0x7fff7fffu);
  return __vmaxu2(m, v.w & 0x7fff7fffu);
}

// what an edge or whole block has to do with
struct PageJob {
  const uint16_t* rows;                                         // new rows of its head, keys or values
  long long stride;
  uint16_t* tail;                                               // the sequence's waiting rows
  int b, h;
  bool keys;
  Seq q;
};
__device__ __forceinline__ PageJob page_job(const AppendArgs& a, int b, int h, bool keys, const Seq& q) {
  const uint16_t* rows = (keys ? a.k : a.v) + (size_t)h * a.D;
  uint16_t* tail = (keys ? a.k_tail : a.v_tail) + ((size_t)b * a.Hkv + h) * a.s.page * a.D;
  return PageJob{rows, keys ? a.ks : a.vs, tail, b, h, keys, q};
}
// unit u of the row at position p of the sequence; new rows of keys are rotated
template <int MODE>
__device__ __forceinline__ void load_unit(const AppendArgs& a, const qp_rope& rope, const uint64_t* turn, const PageJob& w, int p, int u, uint4& x,
                                          uint4& y, int& c0, int& c1) {
  const int rot = rope.rot_dim;
  const bool fresh = p >= w.q.len;
  const int r = w.q.row0 + p - w.q.len;
  const uint16_t* row = fresh ? w.rows + r * w.stride : w.tail + (p & (a.s.page - 1)) * a.D;
  unit_vectors(MODE, rot, u, c0, c1);
  x = *reinterpret_cast<const uint4*>(row + 8 * c0);
  y = *reinterpret_cast<const uint4*>(row + 8 * c1);
  if (fresh && w.keys && rot) {
    const int at = a.pos ? __ldg(a.pos + r) : p;
    rotate_unit<MODE>(x, y, u, rot, row, [&](int j) {
      const float2 c = cos_sin(turn[j], at, rope.factor), d = cos_sin(turn[min(j + 1, (rot >> 1) - 1)], at, rope.factor);
      return make_float4(c.x, c.y, d.x, d.y);
    });
  }
}
// stores page pg of the sequence; all of the block, which meets at a barrier after every row has been read
template <int UNITS, int MODE>
__device__ __forceinline__ void store_page(const AppendArgs& a, const qp_rope& rope, const uint64_t* turn, uint32_t* s_max, const PageJob& w, int pg) {
  const int D = a.D, lgu = D == 128 ? 3 : 2, lgp = 31 - __clz(a.s.page), tid = threadIdx.x;
  const int id = page_of(a.s, w.b, pg);
  uint4 x[UNITS], y[UNITS];
  uint32_t m = 0u;
#pragma unroll
  for (int k = 0; k < UNITS; ++k) {
    const int j = tid + k * THREADS;
    int c0, c1;
    load_unit<MODE>(a, rope, turn, w, (pg << lgp) + (j >> lgu), j & ((1 << lgu) - 1), x[k], y[k], c0, c1);
    m = abs_max2(abs_max2(m, x[k]), y[k]);
  }
  m = max(m & 0xffffu, m >> 16);
  m = __reduce_max_sync(0xffffffffu, m);
  if ((tid & 31) == 0) s_max[tid >> 5] = m;
  __syncthreads();
  m = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
  // the scale is rounded up to bf16, so that no code is cut off; a number that is none makes the whole page so
  const bool e4m3 = a.format == QP_E4M3;
  const float top = __uint_as_float(m << 16);
  const uint32_t sb = m > 0x7f80u ? 0x7fc0u : (__float_as_uint(__fdiv_rn(top, e4m3 ? 448.f : 127.f)) + 0xffffu) >> 16;
  const float sc = __uint_as_float(sb << 16), inv = sc == 0.f ? 0.f : fminf(__fdiv_rn(1.f, sc), FLT_MAX);
  if (id < 0) return;
  const size_t ph = (size_t)id * a.Hkv + w.h;
  uint8_t* codes = (w.keys ? a.kc : a.vc) + (ph << lgp) * D;
  if (tid == 0) (w.keys ? a.k_scale : a.v_scale)[ph] = (uint16_t)sb;
#pragma unroll
  for (int k = 0; k < UNITS; ++k) {
    const int j = tid + k * THREADS;
    int c0, c1;
    unit_vectors(MODE, rope.rot_dim, j & ((1 << lgu) - 1), c0, c1);
    uint8_t* row = codes + (j >> lgu) * D;
    *reinterpret_cast<uint2*>(row + 8 * c0) = codes8(x[k], inv, e4m3);
    *reinterpret_cast<uint2*>(row + 8 * c1) = codes8(y[k], inv, e4m3);
  }
}

// The sequence that a unit of whole pages, or a row, is taken to belong to.
__device__ __forceinline__ int unit_owner(const StepView& s, int unit) {
  const int lgp = 31 - __clz(s.page);
  return last_at_most(s.start, s.n_seqs, unit, [&](int x) { return x >> lgp; });
}
__device__ __forceinline__ int row_owner(const StepView& s, int r) {
  return last_at_most(s.start, s.n_seqs, r, [](int x) { return x; });
}
__device__ __forceinline__ bool has_row(const Seq& q, int r) { return q.n > 0 && r >= q.row0 && r < q.row0 + q.n; }

// Where start falls, those searches can miss the sequence that a unit or a row belongs to, and no block of theirs does the work.  The
// sequence before the first fall is one that is left out, and its edge blocks do it instead: each for its KV head (and keys or values),
// sequence by sequence.  Slow, and never met by a step whose numbers belong together.
template <int UNITS, int MODE>
__device__ __noinline__ void append_missed(const AppendArgs& a, const qp_rope& rope, const uint64_t* turn, uint32_t* s_max, int fall, int h, bool keys) {
  const StepView& s = a.s;
  const int page = s.page, lgp = 31 - __clz(page), lgu = a.D == 128 ? 3 : 2, G = a.Hq / a.Hkv, rot = rope.rot_dim, tid = threadIdx.x;
  for (int b = 0; b < fall; ++b)
    if (__ldg(s.start + b) > __ldg(s.start + b + 1)) return;    // not the first
  for (int b = 0; b < s.n_seqs; ++b) {
    const Seq q = seq_of(s, b);
    if (q.n == 0) continue;
    const int first = (q.len + page - 1) >> lgp, n = ((q.len + q.n) >> lgp) - first;
    for (int i = 0; i < n; ++i) {
      if (unit_owner(s, (q.row0 >> lgp) + i) == b) continue;
      store_page<UNITS, MODE>(a, rope, turn, s_max, page_job(a, b, h, keys, q), first + i);
      __syncthreads();                                          // (s_max has been read)
    }
  }
  if (!a.q || !keys) return;
  for (long long i0 = 0; i0 < ((long long)s.n_tokens * G) << lgu; i0 += THREADS) {
    const long long i = i0 + tid;
    const int row = (int)(i >> lgu), u = (int)i & ((1 << lgu) - 1), r = row / G, head = h * G + row - r * G;
    bool mine = false;
    Seq q{0, 0, 0};
    if (r < s.n_tokens && !has_row(seq_of(s, row_owner(s, r)), r))
      for (int b = 0; b < s.n_seqs && !mine; ++b) {
        q = seq_of(s, b);
        mine = has_row(q, r);
      }
    uint4 x, y;
    int c0, c1;
    unit_vectors(MODE, rot, u, c0, c1);
    if (mine) {
      const uint16_t* src = a.q + r * a.qs + (long long)head * a.D;
      const int at = a.pos ? __ldg(a.pos + r) : q.len + r - q.row0;
      x = *reinterpret_cast<const uint4*>(src + 8 * c0);
      y = *reinterpret_cast<const uint4*>(src + 8 * c1);
      rotate_unit<MODE>(x, y, u, rot, src, [&](int j) {
        const float2 c = cos_sin(turn[j], at, rope.factor), d = cos_sin(turn[min(j + 1, (rot >> 1) - 1)], at, rope.factor);
        return make_float4(c.x, c.y, d.x, d.y);
      });
    }
    __syncwarp();                                               // (in place: a row's units are one warp's)
    if (mine) {
      uint16_t* dst = a.q_out + ((size_t)r * a.Hq + head) * a.D;
      *reinterpret_cast<uint4*>(dst + 8 * c0) = x;
      *reinterpret_cast<uint4*>(dst + 8 * c1) = y;
    }
  }
}

// A block is one of three kinds:
//   edge    (sequence, head, keys or values): the page that waiting rows and new ones complete together, then the new rows that wait
//   whole   (whole page of new tokens, head, keys or values)
//   query   some tokens' queries
// The edge block reads the waiting rows it uses up before it writes new ones in their place.  A page's numbers stay in registers
// between the search for the largest magnitude and the rounding to codes: page * D / 16 / 128 = UNITS units of 16 channels a thread.
// At most 64 registers up to 4 units, so that eight blocks are on an SM (64 one-token sequences 5.2 -> 3.9 us when taken, 8192 tokens
// with 32 query heads 37.8 -> 33.0 us).
// 8192 tokens with 32 query and 8 KV heads are 35.3 us over changing inputs (185 MB, 5.2 TB/s; 33.8 where a graph writes one cache over
// and over), one token 2.1 us, mostly launch.  Pages of 128 tokens with D = 128 take 8 units a thread, 120 to 148 registers and three
// or four blocks an SM: 51.2 us; PAIR_ODD 138 us with 44 channels.
// The host does not know the sequences' lengths, so it launches a whole-page block for every `page` rows of the step: unit u belongs
// to the last sequence b with start[b] / page <= u, which has at least as many of them as pages begin and end in its new tokens.
// Numbers that do not belong together leave out their own sequence only, see append_missed.
template <int UNITS, int MODE, int ROT_UNITS>
__global__ void __launch_bounds__(THREADS, UNITS <= 4 ? 8 : 1)
append_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ qp_rope rope, int edge_blocks, int page_blocks, int tokens,
              uint32_t inv_h) {
  __shared__ __align__(16) float2 table[ROT_TOKENS * 64];
  __shared__ int s_pos[ROT_TOKENS];
  __shared__ uint32_t s_max[THREADS / 32];
  __shared__ uint64_t turn[64];                                 // (each lane reads another: constant memory answers one at a time)
  if (threadIdx.x < rope.rot_dim >> 1) turn[threadIdx.x] = rope.turn[threadIdx.x];
  __syncthreads();
  chain_enter();
  const int bid = blockIdx.x, tid = threadIdx.x;
  const StepView& s = a.s;
  const int D = a.D, lgu = D == 128 ? 3 : 2, page = s.page, lgp = 31 - __clz(page), rot = rope.rot_dim;

  if (bid >= page_blocks) {                                     // queries
    const int t0 = (bid - page_blocks) * tokens, n = min(tokens, s.n_tokens - t0), half = rot >> 1, pitch = table_pitch(rot);
    bool in = false;
    if (tid < n) {
      const int r = t0 + tid;
      const Seq q = seq_of(s, row_owner(s, r));
      in = has_row(q, r);
      s_pos[tid] = a.pos ? __ldg(a.pos + r) : q.len + r - q.row0;
    }
    __shared__ uint32_t s_in;                                   // tokens that are a sequence's
    const uint32_t some = __ballot_sync(0xffffffffu, in);
    if (tid == 0) s_in = some;
    __syncthreads();
    const uint32_t mine = s_in;
    auto fill = [&]() {
      for (int i = tid; i < n * pitch; i += THREADS) {
        const int t = i / pitch, p = i - t * pitch;
        if (p < half) table[t * pitch + table_place(p, pitch)] = cos_sin(turn[p], s_pos[t], rope.factor);
      }
      __syncthreads();
    };
    rotate_tokens<MODE, ROT_UNITS>(a.q + t0 * a.qs, D, a.qs, a.q_out + (size_t)t0 * a.Hq * D, D, (long long)a.Hq * D, n, a.Hq, inv_h, lgu, rot, table, pitch,
                        [&](int t) { return (mine >> t & 1u) != 0; }, fill);
    return;
  }

  const bool edge = bid < edge_blocks;
  const int i = edge ? bid : bid - edge_blocks;
  const bool keys = (i & 1) == 0;
  const int which = (i >> 1) / a.Hkv, h = (i >> 1) - which * a.Hkv;
  int b = which, pg;                                            // sequence, and the page to write (-1: none)
  Seq q;
  if (edge) {
    q = seq_of(s, b);
    pg = q.len >> lgp;
    if (q.len == pg << lgp || q.len + q.n < (pg + 1) << lgp) pg = -1;
    if (q.n == 0 && __ldg(s.start + b) > __ldg(s.start + b + 1)) append_missed<UNITS, MODE>(a, rope, turn, s_max, b, h, keys);
  } else {
    b = unit_owner(s, which);
    q = seq_of(s, b);
    pg = ((q.len + page - 1) >> lgp) + which - (q.row0 >> lgp);
    if (which < q.row0 >> lgp || pg >= (q.len + q.n) >> lgp) return;   // (compared in pages: in tokens it could pass 31 bits)
  }
  if (q.n == 0) return;
  const PageJob w = page_job(a, b, h, keys, q);
  if (pg >= 0) store_page<UNITS, MODE>(a, rope, turn, s_max, w, pg);
  if (edge) {                                                   // (the barrier above: every waiting row of the page has been read)
    const int end = q.len + q.n, lo = max(q.len, end >> lgp << lgp);
    for (int j = tid; j < (end - lo) << lgu; j += THREADS) {
      const int p = lo + (j >> lgu);
      uint4 x, y;
      int c0, c1;
      load_unit<MODE>(a, rope, turn, w, p, j & ((1 << lgu) - 1), x, y, c0, c1);
      uint16_t* row = w.tail + (p & (page - 1)) * D;
      *reinterpret_cast<uint4*>(row + 8 * c0) = x;
      *reinterpret_cast<uint4*>(row + 8 * c1) = y;
    }
  }
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, const qp_rope& rope, cudaStream_t st) {
  const int units = units_a_thread((long long)a.Bt * a.L * a.H, a.D), tokens = tokens_a_block(a.H, a.D, units);
  const dim3 grid((unsigned)(((long long)a.L + tokens - 1) / tokens), std::min(a.Bt, 65535));
  auto launch = [&](auto kernel) { return launch_chained(kernel, grid, dim3(THREADS), 0, st, a, rope, tokens, inverse_of(a.H)); };
  switch (pairing(rope)) {
    case PAIR_NEXT: return units == 4 ? launch(rotary_kernel<PAIR_NEXT, 4>) : launch(rotary_kernel<PAIR_NEXT, 1>);
    case PAIR_HALF: return units == 4 ? launch(rotary_kernel<PAIR_HALF, 4>) : launch(rotary_kernel<PAIR_HALF, 1>);
    default: return units == 4 ? launch(rotary_kernel<PAIR_ODD, 4>) : launch(rotary_kernel<PAIR_ODD, 1>);
  }
}

cudaError_t launch_paged_append(const AppendArgs& a, const qp_rope* rope_or_null, cudaStream_t st) {
  qp_rope rope{};                                               // none: nothing is rotated
  if (rope_or_null) rope = *rope_or_null;
  const int rot_units = units_a_thread((long long)a.s.n_tokens * a.Hq, a.D), tokens = tokens_a_block(a.Hq, a.D, rot_units);
  const long long edge = 2LL * a.s.n_seqs * a.Hkv, whole = 2LL * (a.s.n_tokens / a.s.page) * a.Hkv;
  const long long queries = a.q ? ((long long)a.s.n_tokens + tokens - 1) / tokens : 0;
  if (edge + whole + queries > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)(edge + whole + queries));
  auto launch = [&](auto kernel) {
    return launch_chained(kernel, grid, dim3(THREADS), 0, st, a, rope, (int)edge, (int)(edge + whole), tokens, inverse_of(a.Hq));
  };
#define QP_APPEND(U, M) return rot_units == 4 ? launch(append_kernel<U, M, 4>) : launch(append_kernel<U, M, 1>)
#define QP_APPEND_M(U)                       \
  switch (pairing(rope)) {                   \
    case PAIR_NEXT: QP_APPEND(U, PAIR_NEXT); \
    case PAIR_HALF: QP_APPEND(U, PAIR_HALF); \
    default: QP_APPEND(U, PAIR_ODD);         \
  }
  switch (a.s.page * a.D / 16 / THREADS) {
    case 1: QP_APPEND_M(1)
    case 2: QP_APPEND_M(2)
    case 4: QP_APPEND_M(4)
    case 8: QP_APPEND_M(8)
    default: return cudaErrorInvalidValue;
  }
#undef QP_APPEND_M
#undef QP_APPEND
}

#ifdef QP_CHECKED
cudaError_t rotary_check_read(unsigned int (&out)[4]) { return checked::read_and_clear(out); }
#endif

}  // namespace qp
