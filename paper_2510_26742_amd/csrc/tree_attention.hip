// Attention of drafted tokens over a paged key/value cache (pi0_tree_attention).
//
// All query heads of a key/value head, times all new tokens of a sequence, are rows of one product: K and V are read once
// for all of them.  One pass over the keys in tiles of 32 with a running maximum and sum:
//     S^T = K Q^T  (32 keys x 32 rows, mfma 32x32x16),  p = exp2(scale log2(e) S - m),  O^T += V^T P^T
// S^T leaves a lane one row and 16 of its 32 keys, which is how the second product takes its right operand if the keys
// of a step of 16 are counted as they lie there: probabilities go from one product into the next without leaving their
// lane, row sums and maxima need one exchange between the two halves of a wave.  V^T is read out of row-major tiles with
// the transposing LDS load (4 keys x 16 d per 16 lanes).
// Tiles come straight into LDS, 16 bytes per lane; the pieces of a row are permuted by its key (on the global side: a lane
// may fetch any piece) so that neither product's reads collide in the banks.  Keys without a page or behind the last one are
// fetched from a piece of zeros.
#include "pages_common.h"
#include "exec_ctx.h"

namespace {

typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

__device__ __align__(16) unsigned char zero_piece[16];

template <class T>
struct Mat;
template <>
struct Mat<bf16> {
  static constexpr unsigned EXPONENT = 0x7f80;
  static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mat<f16> {
  static constexpr unsigned EXPONENT = 0x7c00;
  static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

struct TreeArgs {
  pi0_pages p;
  const void* q;
  void* out;
  int64_t q_row_stride, q_head_stride, out_row_stride, out_head_stride;
  int heads, group;      // query heads per key/value head
  const int* row_start;
  int n_rows, max_rows;
  const unsigned* mask;
  int mask_words;
  float scale;           // times log2(e)
  int row_tiles;         // of a sequence and key/value head, at most
  int64_t layer;         // elements in front of the layer
};

// The wave's 32 rows of queries and their running state.  C layout of a 32x32 product: lane = column (row of queries)
// + 32 h, register i = row 8 (i / 4) + 4 h + i % 4.
template <int D>
struct RowState {
  f32x16 o[D / 32];
  float m, l;
};

// T: type; RW waves side by side have 32 rows each, KW of those groups a tile of 32 keys each
template <class T, int D, int RW, int KW>
__global__ __launch_bounds__(64 * RW * KW) void tree_attention_kernel(TreeArgs a) {
  constexpr int PIECES = D / 8, TILE = 32 * D * 2, REQUESTS = TILE / 1024, KEYS_PER_REQUEST = 512 / D;
  constexpr int ROWS = 32 * RW, WAVES = RW * KW;
  const pi0_pages& p = a.p;
  __shared__ __align__(1024) unsigned char tiles[2][KW][TILE];
  unsigned char (*const lds_k)[TILE] = tiles[0];
  unsigned char (*const lds_v)[TILE] = tiles[1];
  __shared__ float weights[WAVES][32][33];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rw = wave % RW, kw = wave / RW, h = lane >> 5;

  const int unit = blockIdx.x;
  const int tile_of_rows = unit % a.row_tiles, kv_head = unit / a.row_tiles % p.kv_heads, seq = unit / a.row_tiles / p.kv_heads;
  const int2 rows = rows_of(a.row_start, seq, a.n_rows, a.max_rows);
  if (tile_of_rows * ROWS >= rows.y * a.group) return;
  const int length = length_of(p, seq), total = min(length + rows.y, p.max_pages * p.page_tokens);

  // this lane's row: token and head
  const int r = tile_of_rows * ROWS + rw * 32 + (lane & 31);
  const bool live = r < rows.y * a.group;
  const int node = live ? r / a.group : 0, head = kv_head * a.group + (live ? r % a.group : 0);
  s16x8 q[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; i++) {
    q[i] = s16x8{};
    if (live)
      q[i] = *reinterpret_cast<const s16x8*>(reinterpret_cast<const T*>(a.q) + (rows.x + node) * a.q_row_stride + head * a.q_head_stride + i * 16 + h * 8);
  }
  const unsigned* mask = a.mask != nullptr ? a.mask + (size_t)(rows.x + node) * a.mask_words : nullptr;

  RowState<D> st;
#pragma unroll
  for (int b = 0; b < D / 32; b++) st.o[b] = f32x16{};
  st.m = -INFINITY;
  st.l = 0.f;

  const int fk_key = lane & 31;
  const int swz_k = (D == 64 ? (fk_key >> 1) & 7 : fk_key & 15) ^ h;
  const int vkey = (lane & 15) >> 2;   // key of a group of four that this lane names in a transposing load
  const int swz_v = D == 64 ? (vkey >> 1) & 1 : vkey;
  const char* const pool_k = reinterpret_cast<const char*>(p.d_k) + 2 * (a.layer + kv_head * p.head_stride);
  const char* const pool_v = reinterpret_cast<const char*>(p.d_v) + 2 * (a.layer + kv_head * p.head_stride);
  const int shift = 31 - __clz(p.page_tokens);

  for (int base = 0; base < total; base += 32 * KW) {
    const int pos0 = base + kw * 32;
    const int page0 = page_at(p, seq, pos0 >> shift), page1 = page_at(p, seq, (pos0 + 16) >> shift);
    __syncthreads();   // the tiles of the round before have been read
#pragma unroll
    for (int j = 0; j < (REQUESTS + RW - 1) / RW; j++) {
      const int request = j * RW + rw;
      if (REQUESTS % RW != 0 && request >= REQUESTS) break;
      const int key = request * KEYS_PER_REQUEST + lane / PIECES, pos = pos0 + key;
      const int page = key < 16 ? page0 : page1;
      const bool there = pos < total && page >= 0;
      const int64_t at = 2 * (page * p.page_stride + (pos & (p.page_tokens - 1)) * p.token_stride);
      const int piece = lane % PIECES;
      const int piece_k = piece ^ (D == 64 ? (key >> 1) & 7 : key & 15);
      const int piece_v = piece ^ (D == 64 ? ((key >> 1) & 1) << 2 : (key & 3) << 2);
      const char* from_k = there ? pool_k + at + piece_k * 16 : reinterpret_cast<const char*>(zero_piece);
      const char* from_v = there ? pool_v + at + piece_v * 16 : reinterpret_cast<const char*>(zero_piece);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_address(lds_k[kw]) + request * 1024), "v"(from_k) : "memory");
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_address(lds_v[kw]) + request * 1024), "v"(from_v) : "memory");
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();

    // S^T
    f32x16 s = {};
    const unsigned char* kt = lds_k[kw] + fk_key * (2 * D);
#pragma unroll
    for (int i = 0; i < D / 16; i++) {
      const s16x8 kf = *reinterpret_cast<const s16x8*>(kt + ((swz_k ^ (2 * i)) << 4));
      s = Mat<T>::mfma(kf, q[i], s);
    }
    // what of the tile the row sees, a bit per key
    unsigned seen = 0xffffffffu;
    const bool drafts = pos0 + 32 > length;
    if (drafts || page0 < 0 || page1 < 0) {
      const int j0 = pos0 - length;   // node at the tile's first key
      if (drafts) {
        unsigned nodes = 0;           // bit b: node max(j0, 0) + b
        const int jn = max(j0, 0);
        if (mask != nullptr) {
          const int word = jn >> 5, off = jn & 31;
          const unsigned lo = word < a.mask_words ? mask[word] : 0, hi = word + 1 < a.mask_words ? mask[word + 1] : 0;
          nodes = (unsigned)(((unsigned long long)hi << 32 | lo) >> off);
        } else {
          const int visible = node - jn + 1;
          nodes = visible >= 32 ? 0xffffffffu : visible > 0 ? (1u << visible) - 1 : 0u;
        }
        const int committed = min(32, max(0, -j0));
        seen = committed >= 32 ? 0xffffffffu : (1u << committed) - 1 | nodes << committed;
        const int have = total - pos0;
        if (have < 32) seen &= have > 0 ? (1u << have) - 1 : 0u;
      }
      if (page0 < 0) seen &= 0xffff0000u;
      if (page1 < 0) seen &= 0x0000ffffu;
    }
    const unsigned bits = seen >> (4 * h);   // bit 8 (i / 4) + i % 4 is register i's key
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; i++) {
      s[i] *= a.scale;
      if (!(bits >> (8 * (i >> 2) + (i & 3)) & 1)) s[i] = -INFINITY;
      top = fmaxf(top, s[i]);
    }
    top = max_xor32(top);
    const float m = fmaxf(st.m, top), safe = m == -INFINITY ? 0.f : m;
    const float keep = __builtin_amdgcn_exp2f(st.m - safe);
    st.m = m;
    st.l *= keep;
#pragma unroll
    for (int b = 0; b < D / 32; b++) st.o[b] *= keep;
    s16x8 pf[2];
#pragma unroll
    for (int i = 0; i < 16; i++) {
      const T w = (T)__builtin_amdgcn_exp2f(s[i] - safe);
      pf[i >> 3][i & 7] = __builtin_bit_cast(short, w);
      st.l += (float)w;   // what the product takes, so that rounding a dominant weight cancels
    }
    const unsigned char* vt = lds_v[kw];
    bool odd_values = false;   // values that a weight of zero does not silence
    if (drafts) {
#pragma unroll
      for (int i = 0; i < TILE / 1024; i++) {
        const uint4 u = *reinterpret_cast<const uint4*>(vt + (i * 64 + lane) * 16);
        const unsigned e = Mat<T>::EXPONENT, word[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int c = 0; c < 4; c++) odd_values |= (word[c] & e) == e || (word[c] >> 16 & e) == e;
      }
    }
    if (__ballot(odd_values) == 0) {
      const unsigned char* lane_v = vt + (4 * h + vkey) * (2 * D) + ((lane >> 4) & 1) * 32 + ((lane & 3) >> 1) * 16 + (lane & 1) * 8;
#pragma unroll
      for (int b = 0; b < D / 32; b++) {
#pragma unroll
        for (int step = 0; step < 2; step++) {
          typedef __attribute__((address_space(3))) s16x4* LdsPtr;
          const unsigned char* at = lane_v + ((b ^ swz_v) << 6) + step * 16 * 2 * D;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(const s16x4*)at);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(const s16x4*)(at + 8 * 2 * D));
          st.o[b] = Mat<T>::mfma(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), pf[step], st.o[b]);
        }
      }
    } else {
      // Rare: a draft's values hold infinities or NaN.  Key by key, and only for the rows that see it.
      float (*wt)[33] = weights[wave];
#pragma unroll
      for (int i = 0; i < 16; i++) {
        const int key = 8 * (i >> 2) + 4 * h + (i & 3);
        const short w = pf[i >> 3][i & 7];
        wt[key][lane & 31] = seen >> key & 1 ? (float)__builtin_bit_cast(T, w) : -1.0f;
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      for (int key = 0; key < 32; key++) {
        const float w = wt[key][lane & 31];
        if (w < 0.f) continue;
        const int swz = D == 64 ? ((key >> 1) & 1) << 2 : (key & 3) << 2;
        const unsigned char* row = vt + key * 2 * D + 8 * h;
#pragma unroll
        for (int c = 0; c < D / 8; c++) {
          const s16x4 v = *reinterpret_cast<const s16x4*>(row + ((c ^ swz) << 4));
#pragma unroll
          for (int i = 0; i < 4; i++) st.o[c >> 2][(c & 3) * 4 + i] += w * (float)__builtin_bit_cast(T, (short)v[i]);
        }
      }
    }
  }
  st.l = add_xor32(st.l);

  // the KW groups' states into the first one's
  if (KW > 1) {
    static_assert(KW == 1 || RW * (D / 2 + 2) * 256 <= 2 * KW * TILE, "a state per row group fits the tiles");
    float* const share = reinterpret_cast<float*>(tiles);   // [RW][D / 32 * 16 + 2][64]; the tiles have been read
    for (int from = 1; from < KW; from++) {
      __syncthreads();
      float* mine = share + rw * (D / 2 + 2) * 64 + lane;
      if (kw == from) {
#pragma unroll
        for (int b = 0; b < D / 32; b++)
#pragma unroll
          for (int i = 0; i < 16; i++) mine[(b * 16 + i) * 64] = st.o[b][i];
        mine[D / 2 * 64] = st.m;
        mine[(D / 2 + 1) * 64] = st.l;
      }
      __syncthreads();
      if (kw == 0) {
        const float om = mine[D / 2 * 64], m = fmaxf(st.m, om), safe = m == -INFINITY ? 0.f : m;
        const float c0 = __builtin_amdgcn_exp2f(st.m - safe), c1 = __builtin_amdgcn_exp2f(om - safe);
        st.m = m;
        st.l = st.l * c0 + mine[(D / 2 + 1) * 64] * c1;
#pragma unroll
        for (int b = 0; b < D / 32; b++)
#pragma unroll
          for (int i = 0; i < 16; i++) st.o[b][i] = st.o[b][i] * c0 + mine[(b * 16 + i) * 64] * c1;
      }
    }
  }
  if (kw != 0 || !live) return;
  const float inv = st.l == 0.f ? 0.f : 1.0f / st.l;
  T* out = reinterpret_cast<T*>(a.out) + (rows.x + node) * a.out_row_stride + head * a.out_head_stride;
#pragma unroll
  for (int b = 0; b < D / 32; b++) {
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      typedef T T4 __attribute__((ext_vector_type(4)));
      T4 w;
#pragma unroll
      for (int c = 0; c < 4; c++) w[c] = (T)(st.o[b][i + c] * inv);
      *reinterpret_cast<T4*>(out + b * 32 + 2 * i + 4 * h) = w;
    }
  }
}

template <class T, int D>
void launch(hipStream_t s, TreeArgs& a) {
  const int most = a.max_rows * a.group;
  if (most <= 32) {
    a.row_tiles = 1;
    hipLaunchKernelGGL((tree_attention_kernel<T, D, 1, 2>), dim3(a.p.n_seqs * a.p.kv_heads), dim3(128), 0, s, a);
  } else {
    a.row_tiles = ceil_div(most, 128);
    hipLaunchKernelGGL((tree_attention_kernel<T, D, 4, 1>), dim3(a.p.n_seqs * a.p.kv_heads * a.row_tiles), dim3(256), 0, s, a);
  }
}

bool args_ok(const pi0_pages* p, int heads, int n_rows, int max_rows) {
  return pages_ok(p) && heads >= 1 && heads <= 1024 && heads % p->kv_heads == 0 && n_rows >= 1 && n_rows <= 1 << 24 && max_rows >= 1 &&
         max_rows <= 1024 && max_rows <= n_rows;
}

}  // namespace

extern "C" {

size_t pi0_tree_attention_workspace_bytes(const pi0_pages* pages, int heads, int n_rows, int max_rows) {
  return args_ok(pages, heads, n_rows, max_rows) ? 16 : 0;
}

int pi0_tree_attention(const pi0_pages* pages, int layer, const pi0_rows* q, const pi0_rows* out, const int32_t* d_row_start, int n_rows,
                       int max_rows, const uint32_t* d_mask, int mask_words, float scale, void* d_workspace, size_t ws_bytes, void* hip_stream) {
  if (q == nullptr || d_row_start == nullptr || ((uintptr_t)d_row_start & 3) != 0 || !args_ok(pages, q->heads, n_rows, max_rows)) return PI0_EINVAL;
  if (layer < 0 || layer >= pages->layers || !(scale - scale == 0.f)) return PI0_EINVAL;
  if (!rows_ok(q, 0, pages->head_dim, pages->dtype) || !rows_ok(out, q->heads, pages->head_dim, pages->dtype)) return PI0_EINVAL;
  if (mask_words < 0 || mask_words > 32 || (mask_words == 0) != (d_mask == nullptr) || ((uintptr_t)d_mask & 3) != 0) return PI0_EINVAL;
  if (d_workspace == nullptr || ((uintptr_t)d_workspace & 15) != 0) return PI0_EINVAL;
  if (ws_bytes < pi0_tree_attention_workspace_bytes(pages, q->heads, n_rows, max_rows)) return PI0_ENOMEM;
  TreeArgs a = {};
  a.p = *pages;
  a.q = q->d_x;
  a.out = out->d_x;
  a.q_row_stride = q->row_stride;
  a.q_head_stride = q->head_stride;
  a.out_row_stride = out->row_stride;
  a.out_head_stride = out->head_stride;
  a.heads = q->heads;
  a.group = q->heads / pages->kv_heads;
  a.row_start = d_row_start;
  a.n_rows = n_rows;
  a.max_rows = max_rows;
  a.mask = d_mask;
  a.mask_words = mask_words;
  a.scale = scale * 1.4426950408889634f;
  a.layer = layer * pages->layer_stride;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const int d = pages->head_dim;
  if (pages->dtype == PI0_BF16) {
    if (d == 64) launch<bf16, 64>(s, a);
    else if (d == 128) launch<bf16, 128>(s, a);
    else launch<bf16, 256>(s, a);
  } else {
    if (d == 64) launch<f16, 64>(s, a);
    else if (d == 128) launch<f16, 128>(s, a);
    else launch<f16, 256>(s, a);
  }
  return hipGetLastError() == hipSuccess ? PI0_OK : PI0_EHIP;
}

}  // extern "C"
