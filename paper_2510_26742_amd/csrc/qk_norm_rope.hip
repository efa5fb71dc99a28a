// Norms of queries and keys for each head, with the position rotation in the same pass; keys and values go into the pages
// of the cache (pi0_qk_norm_rope).
//
// A head of D elements belongs to D / 8 lanes, so a wave holds 2, 4 or 8 heads.  A lane takes two runs of four elements:
// of the rotated part those that pair with each other, (4 l .. , 4 l .. + rope_dim / 2) or, interleaved, eight neighbours; of
// the rest eight neighbours.  So a rotation needs nothing from another lane, and the mean square is a sum over the lanes of
// the head.  The angles' cosines and sines are the same for all heads of a token: a wave computes them once and walks over
// the token's heads.  Bound by memory: every element is read once and written once (8817 tokens of 8 + 1 + 1 heads of 256 in 8 sequences:
// 90 MB in 22 us, 4.1 TB/s; a copy of many times that reaches 4.9); one token by four trips to memory in a row and by its
// code's first fetch (6.8 us).  Reading elements ahead, of the first heads in front of the angles and then of the next heads, gains
// nothing (23.0 and 6.9 us): a unit's other waves fill the time as well.
#include "pages_common.h"

#include <math.h>

namespace {

struct QkvRows {
  const void* x;
  int64_t row_stride, head_stride;
};
struct NormRopeArgs {
  pi0_pages p;
  int layer;
  QkvRows q, k, v;
  void* out;
  int64_t out_row_stride, out_head_stride;
  int heads;
  const int* row_start;
  int n_rows, max_rows;
  const int* position;
  const float* q_gain;
  const float* k_gain;
  float gain_offset, eps;
  int rope_dim, interleaved;
  // turns per position of each pair.  In 64 bits: far positions times a slow frequency keep their fraction of a turn
  double turns[128];
};

typedef float f32x8 __attribute__((ext_vector_type(8)));

template <class X>
__device__ __forceinline__ f32x8 load8(const X* x, int a, int b) {
  typedef X X4 __attribute__((ext_vector_type(4)));
  const X4 u = *reinterpret_cast<const X4*>(x + a), w = *reinterpret_cast<const X4*>(x + b);
  f32x8 r;
#pragma unroll
  for (int i = 0; i < 4; i++) r[i] = (float)u[i], r[4 + i] = (float)w[i];
  return r;
}
template <class T>
__device__ __forceinline__ void store8(T* x, int a, int b, f32x8 v) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 u, w;
#pragma unroll
  for (int i = 0; i < 4; i++) u[i] = (T)v[i], w[i] = (T)v[4 + i];
  *reinterpret_cast<T4*>(x + a) = u;
  *reinterpret_cast<T4*>(x + b) = w;
}

// T: type of the cache and of `out`, X: of q, k and v.  A wave per token
template <class T, class X, int D>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(NormRopeArgs a) {
  const pi0_pages& p = a.p;
  constexpr int LANES = D / 8, HEADS = 64 / LANES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int seq = blockIdx.y, token = blockIdx.x * 4 + wave;
  const int2 rows = rows_of(a.row_start, seq, a.n_rows, a.max_rows);
  if (token >= rows.y) return;
  const int row = rows.x + token, l = lane % LANES;
  const int place = length_of(p, seq) + token;
  const int page = page_at(p, seq, place / p.page_tokens);
  const int64_t at_token = a.layer * p.layer_stride + page * p.page_stride + (place % p.page_tokens) * p.token_stride;

  const bool turned = 8 * l < a.rope_dim;
  const int first = !turned || a.interleaved ? 8 * l : 4 * l;
  const int second = !turned || a.interleaved ? first + 4 : first + a.rope_dim / 2;
  float cs[4], sn[4];
  if (turned) {
    const double where = (double)(a.position != nullptr ? a.position[row] : place);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const double turns = where * a.turns[4 * l + i];
      sincospif(2.0f * (float)(turns - rint(turns)), &sn[i], &cs[i]);
    }
  }
  f32x8 q_gain = {1, 1, 1, 1, 1, 1, 1, 1}, k_gain = q_gain;
  if (a.q_gain != nullptr) q_gain = load8(a.q_gain, first, second) + a.gain_offset;
  if (a.k_gain != nullptr) k_gain = load8(a.k_gain, first, second) + a.gain_offset;

  const int all = a.heads + 2 * p.kv_heads;
  for (int base = 0; base < all; base += HEADS) {
    const int h = base + lane / LANES, kh = h - a.heads, vh = kh - p.kv_heads;
    const bool is_q = h < a.heads, is_k = !is_q && kh < p.kv_heads, is_v = h < all && !is_q && !is_k;
    f32x8 x = {};
    if (is_q) x = load8(reinterpret_cast<const X*>(a.q.x) + row * a.q.row_stride + h * a.q.head_stride, first, second);
    if (is_k) x = load8(reinterpret_cast<const X*>(a.k.x) + row * a.k.row_stride + kh * a.k.head_stride, first, second);
    if (is_v) x = load8(reinterpret_cast<const X*>(a.v.x) + row * a.v.row_stride + vh * a.v.head_stride, first, second);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) sum += x[i] * x[i];
#pragma unroll
    for (int i = 1; i < LANES; i <<= 1) sum += __shfl_xor(sum, i);
    f32x8 y = x;
    if (is_q ? a.q_gain != nullptr : is_k && a.k_gain != nullptr) {
      const float rms = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
      y = x * rms * (is_q ? q_gain : k_gain);
    }
    if (turned && !is_v) {
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const float u = y[2 * i], w = y[2 * i + 1];
          y[2 * i] = u * cs[i] - w * sn[i];
          y[2 * i + 1] = u * sn[i] + w * cs[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const float u = y[i], w = y[4 + i];
          y[i] = u * cs[i] - w * sn[i];
          y[4 + i] = u * sn[i] + w * cs[i];
        }
      }
    }
    if (is_q) store8(reinterpret_cast<T*>(a.out) + row * a.out_row_stride + h * a.out_head_stride, first, second, y);
    if (is_k && page >= 0) store8(reinterpret_cast<T*>(p.d_k) + at_token + kh * p.head_stride, first, second, y);
    if (is_v && page >= 0) store8(reinterpret_cast<T*>(p.d_v) + at_token + vh * p.head_stride, first, second, y);
  }
}

template <class T, class X, int D>
hipError_t launch(hipStream_t s, const NormRopeArgs& a) {
  return enqueue(s, dim3(div_up(a.max_rows, 4), a.p.n_seqs), 256, qk_norm_rope_kernel<T, X, D>, a);
}
template <class T, class X>
hipError_t launch_dim(hipStream_t s, const NormRopeArgs& a) {
  if (a.p.head_dim == 64) return launch<T, X, 64>(s, a);
  if (a.p.head_dim == 128) return launch<T, X, 128>(s, a);
  return launch<T, X, 256>(s, a);
}

}  // namespace

extern "C" int pi0_qk_norm_rope(const pi0_pages* pages, int layer, const pi0_rows* q, const pi0_rows* k, const pi0_rows* v, const pi0_rows* out,
                                const int32_t* d_row_start, int n_rows, int max_rows, const int32_t* d_position, const float* d_q_gain,
                                const float* d_k_gain, float gain_offset, float eps, int rope_dim, double rope_base, int interleaved,
                                void* hip_stream) {
  if (!pages_ok(pages) || layer < 0 || layer >= pages->layers || q == nullptr || d_row_start == nullptr) return PI0_EINVAL;
  const int d = pages->head_dim, type = q->dtype;
  if (type != PI0_F32 && type != pages->dtype) return PI0_EINVAL;
  if (!rows_ok(q, 0, d, type) || !rows_ok(k, pages->kv_heads, d, type) || !rows_ok(v, pages->kv_heads, d, type) ||
      !rows_ok(out, q->heads, d, pages->dtype))
    return PI0_EINVAL;
  if (n_rows < 1 || n_rows > 1 << 24 || max_rows < 1 || max_rows > n_rows) return PI0_EINVAL;
  if ((((uintptr_t)d_q_gain | (uintptr_t)d_k_gain) & 15) != 0 || ((uintptr_t)d_row_start & 3) != 0 || ((uintptr_t)d_position & 3) != 0) return PI0_EINVAL;
  if (rope_dim < 0 || rope_dim > d || rope_dim % 8 != 0 || !(eps >= 0.f)) return PI0_EINVAL;
  if (rope_dim > 0 && !(rope_base > 0.0 && rope_base < HUGE_VAL)) return PI0_EINVAL;
  NormRopeArgs a = {};
  a.p = *pages;
  a.layer = layer;
  a.q = {q->d_x, q->row_stride, q->head_stride};
  a.k = {k->d_x, k->row_stride, k->head_stride};
  a.v = {v->d_x, v->row_stride, v->head_stride};
  a.out = out->d_x;
  a.out_row_stride = out->row_stride;
  a.out_head_stride = out->head_stride;
  a.heads = q->heads;
  a.row_start = d_row_start;
  a.n_rows = n_rows;
  a.max_rows = max_rows;
  a.position = d_position;
  a.q_gain = d_q_gain;
  a.k_gain = d_k_gain;
  a.gain_offset = gain_offset;
  a.eps = eps;
  a.rope_dim = rope_dim;
  a.interleaved = interleaved != 0;
  // base^(-2 i / rope_dim): as exp, a quarter of pow's time; the rounding of its argument a costs a e^-a 2^-53 <= 2^-54 of a turn per position
  const double step = rope_dim > 0 ? -2.0 * log(rope_base) / rope_dim : 0.0;
  for (int i = 0; i < rope_dim / 2; i++) a.turns[i] = exp(i * step) / (2.0 * M_PI);
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  hipError_t e;
  if (pages->dtype == PI0_BF16) e = type == PI0_F32 ? launch_dim<bf16, float>(s, a) : launch_dim<bf16, bf16>(s, a);
  else e = type == PI0_F32 ? launch_dim<f16, float>(s, a) : launch_dim<f16, f16>(s, a);
  return e == hipSuccess ? PI0_OK : PI0_EHIP;
}
