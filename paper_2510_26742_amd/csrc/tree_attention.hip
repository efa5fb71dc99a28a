// Attention of drafted tokens over a paged key/value cache (pi0_tree_attention).
//
// All query heads of a key/value head, times all new tokens of a sequence, are rows of one product: K and V are read once
// for all of them.  One pass over the keys, 32 at a time, with a running maximum and sum:
//     S^T = K Q^T  (16 keys x 16 rows, mfma 16x16x32),  p = exp2(scale log2(e) S - m),  O^T += V^T P^T
// S^T leaves a lane one row and 4 of 16 keys, which is how the second product takes its right operand if the keys of its 32
// are counted as they lie there: probabilities go from one product into the next without leaving their lane, row sums and
// maxima need two exchanges between the quarters of a wave.  V^T is read out of row-major tiles with the transposing LDS
// load (4 keys x 16 d per 16 lanes).  A wave has R times 16 rows: what it reads of K and V out of LDS serves all of them.  R = 1 where
// the cache's own bytes are what the time goes to, 2 where rows are many.
// What bounds it: few rows the reads of the cache (64 x 1 token, 8 heads over 1 of 256, up to 8192 keys: 277 MB in 43.4 us, 6.4 TB/s);
// many rows what a wave that is alone on its SIMD does one after the other (8 x 64 nodes over 16384: 25.8 GFLOP in 47.4 us, 545 TFLOP/s).  A
// granule takes it 2370 cycles: scores with weights and requests beside them 1070, sums with maxima 790, the barrier and the looks at what is to be cleaned,
// hidden and rescaled the rest.  Its 64 products could end in 1024 (the matrix cores are busy 30 % of the kernel's time); its reads of shared memory
// take 1150 (without conflicts 31 cycles per 16 bytes a lane, 21 per transposing read), its 350 instructions 1400 to issue.  28 granules are 66 of a
// wave's 87 thousand cycles, the beginning and partial results the others.
// Tiles come straight into LDS, 16 bytes per lane; the pieces of a row are permuted by its key (on the global side: a lane
// may fetch any piece) so that neither product's reads collide in the banks.
#include "pages_common.h"
#include "exec_ctx.h"

#include <type_traits>

namespace {

typedef f16 f16x2 __attribute__((ext_vector_type(2)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

template <class T>
struct Mat;
template <>
struct Mat<bf16> {
  static constexpr unsigned EXPONENT = 0x7f80;
  static __device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mat<f16> {
  static constexpr unsigned EXPONENT = 0x7c00;
  static __device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

// How the work is cut.  A unit is a tile of 64 R rows of one sequence and key/value head against all of its keys, in granules of 32
// keys.  Lengths differ, and the host does not know them, so every block works out from the lengths which granules are its
// own: the units lie behind each other on a line that is cut into runs of equal length, one per block.  A unit is START granules longer
// than it is - what a block spends before a unit's first granule and behind its last -, and a run, LEAST long at least, may end one
// unit, hold others and begin the next.  A block writes a unit that it has all of; of any other it leaves a partial result, in slot 1 if it
// has the first granule, in slot 0 if not, and the second launch joins them.
// LEAST: of few keys, runs of 1 or 2 make more partial results than their reading at once is worth (4 x 8 tokens over up to 4096, 8 heads over
// 1 of 256: 19.6 us with 1, 15.2 with 2, 14.1 with 3), long ones take their time one granule behind the other (1 token over 816: 8.7, 9.5, 9.4, with 4
// 10.9).  A tile that is full, 64 rows or more, has partial results of twice and four times the bytes: LEAST_FULL (1 x 16 over 1024 / 4096 / 16384
// 11.8 / 14.1 / 21.8 us with 3, 11.9 / 13.7 / 20.3 with 4, 13.9 / 14.5 / 18.4 with 6; of 84 such cases the mean is 18.3, 18.0, 18.1).
// START: 12 costs short units up to 4 %, 2 lets row tiles of the same keys drift apart, so that each fetches them for itself (8 x 64 over
// 16384 in tiles of 64 rows: 75.8 us with 2, 61.9 with 6).
constexpr int GRANULE = 32, START = 6, LEAST = 3, LEAST_FULL = 4;

// A stage of K and V tiles is 128 D bytes; STAGES of them per block.  BLOCKS: as many as the chip's 256 compute units hold at once, two
// to each where registers let them: one reads while another begins or ends a unit or waits for its waves.  Heads of 64 have so little
// work per granule that four pay (64 x 1 over up to 4096, 8 heads over 8: 78.6 us with two, 59.3 with three, 53.0 with four, 79.0 with
// two of 8 stages; the most that it costs is 4 x 16 over 16384, 8 over 1: 15.7, 16.7, 18.4); those of 128 are as fast with three
// of 3 stages as with two of 4 (117 us).
// Blocks of 1 or 2 waves for few rows are no faster than those of 4 with a wave or two that only request (64 x 1 over up to 8192, 8
// heads over 1 of 256: 53.3, 52.0, 51.5 us; 1 over 816: 9.8, 9.0, 8.7).
template <int D, int R>
struct Shape;
template <> struct Shape<256, 1> { static constexpr int STAGES = 2, BLOCKS = 512; };
template <> struct Shape<256, 2> { static constexpr int STAGES = 4, BLOCKS = 256; };
template <> struct Shape<128, 1> { static constexpr int STAGES = 4, BLOCKS = 512; };
template <> struct Shape<128, 2> { static constexpr int STAGES = 4, BLOCKS = 512; };
template <> struct Shape<64, 1> { static constexpr int STAGES = 4, BLOCKS = 1024; };
template <> struct Shape<64, 2> { static constexpr int STAGES = 4, BLOCKS = 512; };

// a unit's share of the line
__device__ __forceinline__ int share_of(int granules) { return granules > 0 ? granules + START : 0; }

struct TreeArgs {
  pi0_pages p;
  const void* q;
  void* out;
  int64_t q_row_stride, q_head_stride, out_row_stride, out_head_stride;
  int group;             // query heads per key/value head
  const int* row_start;
  int n_rows, max_rows;
  const unsigned* mask;
  int mask_words;
  float scale;           // times log2(e), > 0
  int odd_scale;         // it was not: the queries' signs are turned (negate) or all of their bits cleared (q_bits)
  short negate, q_bits;
  int64_t layer;         // elements in front of the layer
  // workspace
  int* upto;             // [n_seqs] where a sequence's share of the line ends
  int* run;              // granules per run
  f32x4* part_o;         // [runs][2][sets][head_dim / 16][64]: as a wave holds them
  float2* part_ml;       // [runs][2][sets][16]: reference of the exponents, sum of the weights
  int sets;              // of 16 rows in a tile, or in all there are
};

// A sequence's entry idx, the same for the whole wave: through the scalar cache, so that it does not wait in line behind the tiles
// that are on their way
__device__ __forceinline__ int entry_at(const pi0_pages& p, int seq, int idx) {
  return ((const __attribute__((address_space(4))) int*)p.d_table)[(size_t)seq * p.max_pages + min(idx, p.max_pages - 1)];
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Reads of tiles by LDS address.  A tile's rows are 2 D bytes, its pieces permuted by an exclusive or with the key, so the address
// of piece c is that of piece 0 of the same lane with bits turned over.
typedef const __attribute__((address_space(3))) s16x8* LdsPiece;
typedef __attribute__((address_space(3))) s16x4* LdsQuad;

// S^T has a lane own one row of queries: lane = column (row of queries) + 16 quad, register i = key 4 quad + i; O^T the same with d in
// the place of keys.
template <int D>
struct RowState {
  f32x4 o[D / 16];
  float m, l;    // reference of the exponents, sum of this lane's weights
  float shift;   // -m, 0 where that is infinite
};

__device__ __forceinline__ float dot_ones(bf16x2 w, float c) { return __builtin_amdgcn_fdot2_f32_bf16(w, bf16x2{(bf16)1.0f, (bf16)1.0f}, c, false); }
__device__ __forceinline__ float dot_ones(f16x2 w, float c) { return __builtin_amdgcn_fdot2(w, f16x2{(f16)1.0f, (f16)1.0f}, c, false); }

// o *= c, where it is: in the accumulation registers.  Written as a product, the sums are copied to vector registers in every granule, whether
// or not the branch is taken (64 instructions at D = 256).  The products that wrote them may stand right in front: the wait
// there, 64 cycles, is several times what the last of them takes, the one behind covers a product that reads what was written.
template <int N>
__device__ __forceinline__ void scale_sums(f32x4 (&o)[N], float c) {
  asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
  for (int b = 0; b < N; b++) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      float x = o[b][i], t;
      asm volatile("v_accvgpr_read_b32 %1, %0\n\tv_mul_f32 %1, %1, %2\n\tv_accvgpr_write_b32 %0, %1" : "+a"(x), "=&v"(t) : "v"(c));
      o[b][i] = x;
    }
  }
  asm volatile("s_nop 15" ::: "memory");
}

// whether 16 bytes of LDS hold an infinity or a NaN; CLEAN: puts zeros in their place
template <class T, bool CLEAN>
__device__ __forceinline__ bool clean(unsigned char* at) {
  constexpr unsigned E = Mat<T>::EXPONENT;
  uint4 u = *reinterpret_cast<const uint4*>(at);
  unsigned word[4] = {u.x, u.y, u.z, u.w};
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const bool lo = (word[i] & E) == E, hi = (word[i] >> 16 & E) == E;
    odd |= lo || hi;
    word[i] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0x0000ffffu : ~0u);
  }
  if (CLEAN && odd) *reinterpret_cast<uint4*>(at) = uint4{word[0], word[1], word[2], word[3]};
  return odd;
}

// another lane's value by a data-parallel move (CTRL as the hardware counts them), 0 where there is none; ROWS: of 16 lanes that take part
template <int CTRL, int ROWS = 0xf, class V>
__device__ __forceinline__ V dpp(V v) {
  return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ int wave_prefix(int v) {   // sum over the lanes up to this one
  v += dpp<0x111>(v);   // lanes 1, 2, 4, 8 below, inside rows of 16; then the rows' last lanes to the rows behind
  v += dpp<0x112>(v);
  v += dpp<0x114>(v);
  v += dpp<0x118>(v);
  v += dpp<0x142, 0xa>(v);
  v += dpp<0x143, 0xc>(v);
  return v;
}

// 4 waves of a block have R times 16 rows each and read the same tiles
constexpr int RW = 4;
template <class T, int D, int R>
__global__ __launch_bounds__(64 * RW, D < 256 || R == 1 ? 2 : 1) void tree_attention_kernel(TreeArgs a) {
  constexpr int STAGES = Shape<D, R>::STAGES, BLOCKS = Shape<D, R>::BLOCKS, ROWS = 16 * R * RW;
  constexpr int PIECES = D / 8, TILE = 32 * D * 2, PARTS = TILE / 1024, REQUESTS = 2 * PARTS / RW, KEYS_PER_REQUEST = 512 / D;
  constexpr int AHEAD = R > 1;
  constexpr int STEPS = D / 32, TILES = D / 16;   // of 32 d that scores are summed over, of 16 d that sums are kept for
  static_assert(REQUESTS >= 1 && STAGES >= (AHEAD ? 3 : 2) && (STAGES - 2) * REQUESTS < 64, "the wait counter holds what is in flight");
  typedef T T2 __attribute__((ext_vector_type(2)));
  typedef T T4 __attribute__((ext_vector_type(4)));
  const pi0_pages& p = a.p;
  __shared__ __align__(1024) unsigned char tiles[STAGES][2][TILE];
  __shared__ int end_of[MAX_SEQS];   // where a sequence's share of the line ends
  const int lane = threadIdx.x & 63, rw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quad = lane >> 4;

  // The line, worked out by every wave for itself: lane l has the sequences l, l + 64, ..; what it knows of the first 64 stays in
  // registers.  (Whatever runs once per block is written to be short: a block starts with its code far away, and 64 bytes
  // of it cost about as long as a read of memory that is near.)
  int line, my_end = 0, run;
  int2 my_rows = {0, 0};
  int my_length = 0;
  {
    int before = 0;
#pragma unroll 1
    for (int s0 = 0; s0 < p.n_seqs; s0 += 64) {
      const int s = s0 + lane;
      int2 rows = {0, 0};
      int length = 0;
      if (s < p.n_seqs) rows = rows_of(a.row_start, s, a.n_rows, a.max_rows), length = length_of(p, s);
      const int units = p.kv_heads * div_up(rows.y * a.group, ROWS), granules = div_up(min(length + rows.y, p.max_pages * p.page_tokens), GRANULE);
      const int end = before + wave_prefix(units * share_of(granules));
      if (s0 == 0) my_rows = rows, my_length = length;
      if (s0 == 0) my_end = end;
      if (rw == 0 && s < p.n_seqs) {
        end_of[s] = end;
        if (blockIdx.x == 0) a.upto[s] = end;
      }
      before = __builtin_amdgcn_readlane(end, 63);
    }
    line = before;
    run = max(a.sets < 4 ? LEAST : LEAST_FULL, div_up(line, BLOCKS));
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.run = run;
    if (p.n_seqs > 64) __syncthreads();
  }
  const int begin = (int)min((int64_t)line, (int64_t)blockIdx.x * run), end = (int)min((int64_t)line, (int64_t)begin + run);

  // This lane's pieces.  First product: keys lane % 16 and that + 16, pieces quad, quad + 4, ..; second: of 4 keys and 16 d that 16
  // lanes read transposed, key (lane % 16) / 4 and 4 d of lane % 4.  Requests: row lane / PIECES of a KiB, its piece lane % PIECES -
  // where the row's permuted piece lies in the cache.
  const int kkey = lane & 15, vkey = 4 * quad + (kkey >> 2);
  const unsigned read_k = kkey * 2 * D + (((D == 64 ? kkey >> 1 : kkey) ^ quad) << 4);
  const unsigned read_v = vkey * 2 * D + ((D == 64 ? (vkey >> 1) & 3 : vkey & 7) << 5) + (lane & 3) * 8;
  const int my_row = lane / PIECES, my_piece = lane % PIECES;
  const int piece_k0 = my_piece ^ (D == 64 ? (my_row >> 1) & 7 : my_row), piece_v0 = my_piece ^ ((D == 64 ? (my_row >> 1) & 3 : my_row) << 1);
  const int shift = 31 - __clz(p.page_tokens), in_page = p.page_tokens - 1;
  const unsigned lds0 = lds_address(&tiles[0][0][0]);

  for (int cur = begin; cur < end;) {
    // the unit that this run is in
    int seq = 0, before, length;
    int2 rows;
    if (p.n_seqs <= 64) {
      seq = __popcll(__ballot(lane < p.n_seqs && my_end <= cur));
      before = seq > 0 ? __builtin_amdgcn_readlane(my_end, seq - 1) : 0;
      rows.x = __builtin_amdgcn_readlane(my_rows.x, seq);
      rows.y = __builtin_amdgcn_readlane(my_rows.y, seq);
      length = __builtin_amdgcn_readlane(my_length, seq);
    } else {
      for (int top = p.n_seqs - 1; seq < top;) {
        const int mid = (seq + top) >> 1;
        if (end_of[mid] <= cur) seq = mid + 1;
        else top = mid;
      }
      seq = uniform(seq);
      before = uniform(seq > 0 ? end_of[seq - 1] : 0);
      rows = rows_of(a.row_start, seq, a.n_rows, a.max_rows);
      rows.x = uniform(rows.x), rows.y = uniform(rows.y);
      length = uniform(length_of(p, seq));
    }
    const int total = min(length + rows.y, p.max_pages * p.page_tokens), granules = div_up(total, GRANULE), row_tiles = div_up(rows.y * a.group, ROWS);
    const int share = granules + START, inside = cur - before, room = share * row_tiles;   // of a key/value head
    const int kv_head = p.kv_heads > 1 ? (unsigned)inside / (unsigned)room : 0, in_head = inside - kv_head * room;
    const int row_tile = row_tiles > 1 ? (unsigned)in_head / (unsigned)share : 0;
    const int first = before + kv_head * room + row_tile * share + START, g0 = max(0, cur - first), g1 = min(granules, end - first);
    cur = first + granules;
    if (g0 >= g1) continue;   // the run ends in front of the unit's first granule

    // The pages of the first granules.  With AHEAD the last granule is requested again where there is none behind it, into a stage that
    // nobody reads any more: as many requests are on their way at the end as anywhere, and no branch parts the products.
    int entry0, entry1, entries[STAGES - 1][2];
    auto in_unit = [&](int granule) { return AHEAD ? min(granule, g1 - 1) : granule; };
    auto next_entries = [&](int granule) {
      entry0 = entry_at(p, seq, granule * GRANULE >> shift), entry1 = entry_at(p, seq, (granule * GRANULE + 16) >> shift);
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; i++) {
      next_entries(in_unit(g0 + i));
      entries[i][0] = entry0, entries[i][1] = entry1;
    }
    // this lane's rows: token and head
    int node[R], head[R];
    bool live[R];
    const unsigned* mask[R];
    // A lane without a row takes its tile's last one and gives nothing back: scores that its wave has anyway, so it moves no reference of the
    // others, and no other block's row, which may be its result by now (out may be q).
    s16x8 q[R][STEPS];
#pragma unroll
    for (int n = 0; n < R; n++) {
      const int place = row_tile * ROWS + (rw * R + n) * 16 + kkey, r = min(place, rows.y * a.group - 1);
      live[n] = place == r;
      // r / group: both below 2^20, and half a row is more than the reciprocal is off by
      node[n] = (int)(((float)r + 0.5f) * __builtin_amdgcn_rcpf((float)a.group));
      head[n] = kv_head * a.group + r - node[n] * a.group;
      mask[n] = a.mask + (size_t)(rows.x + node[n]) * a.mask_words;
      const T* const q_row = reinterpret_cast<const T*>(a.q) + (rows.x + node[n]) * a.q_row_stride + head[n] * a.q_head_stride + quad * 8;
#pragma unroll
      for (int i = 0; i < STEPS; i++) q[n][i] = *reinterpret_cast<const s16x8*>(q_row + i * 32);
    }
    const char* const pool_k = reinterpret_cast<const char*>(p.d_k) + 2 * (a.layer + kv_head * p.head_stride);
    const char* const pool_v = reinterpret_cast<const char*>(p.d_v) + 2 * (a.layer + kv_head * p.head_stride);

    // Requests of this wave's part of a granule, of whose keys the first and last 16 lie in pages page0 and page1.  Where there is no page
    // (-1), and behind the last position, some row is read that the scores then hide.  A quarter of a granule is 16 keys, or the
    // values of 16: one for each wave.
    constexpr int QUARTER = PARTS / 2;   // KiB
    const bool of_v = rw >= 2;
    struct Quarter {
      const char* from;
      unsigned to;
    };
    auto quarter_of = [&](int granule, int stage, int page0, int page1) {
      const int pos = granule * GRANULE + (rw & 1) * 16, page = max(rw & 1 ? page1 : page0, 0);
      const uint64_t in = (uint64_t)(unsigned)(pos & in_page) * (unsigned)p.token_stride;
      return Quarter{(of_v ? pool_v : pool_k) + 2 * (page * p.page_stride + in), lds0 + stage * 2 * TILE + rw * QUARTER * 1024};
    };
    // 4 KiB (of heads of 64: 2) at once: the instruction's offset counts on both sides, so the LDS address is set once.  (Rows are no
    // less than a head's bytes apart: what is taken off for it is there.  15 strides and a row fit 32 bits.)
    constexpr int BURST = QUARTER < 4 ? QUARTER : 4;
    auto request_burst = [&](const Quarter& at, int burst) {
      unsigned off[BURST];
#pragma unroll
      for (int i = 0; i < BURST; i++) {
        // how far the first key's number turns the pieces of its row (the rest is in piece0)
        const int key = (burst * BURST + i) * KEYS_PER_REQUEST, turn_k = D == 64 ? key >> 1 & 7 : key, turn_v = D == 64 ? 0 : (key & 7) << 1;
        off[i] = (my_row + key) * (unsigned)(2 * p.token_stride) + ((of_v ? piece_v0 : piece_k0) ^ (of_v ? turn_v : turn_k)) * 16 - i * 1024;
      }
      if constexpr (BURST == 2)
        asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:%5"
                     ::"s"(at.to), "v"(off[0]), "v"(off[1]), "s"(at.from), "n"(burst * BURST * 1024), "n"(1024) : "memory", "scc");
      else
        asm volatile("s_add_u32 m0, %0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:%7\n\t"
                     "global_load_lds_dwordx4 %3, %5 offset:%8\n\tglobal_load_lds_dwordx4 %4, %5 offset:%9"
                     ::"s"(at.to), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(at.from), "n"(burst * BURST * 1024), "n"(1024), "n"(2 * 1024),
                     "n"(3 * 1024) : "memory", "scc");
    };
    auto request = [&](int granule, int stage, int page0, int page1) {
      const Quarter at = quarter_of(granule, stage, page0, page1);
#pragma unroll
      for (int burst = 0; burst < QUARTER / BURST; burst++) request_burst(at, burst);
    };

    RowState<D> st[R];
#pragma unroll
    for (int n = 0; n < R; n++) {
#pragma unroll
      for (int b = 0; b < TILES; b++) {
        st[n].o[b] = Mat<T>::mfma(s16x8{}, s16x8{}, f32x4{});   // (zeros, 8 bytes of code for 4 registers)
        asm volatile("" : "+a"(st[n].o[b]));   // (where they stay; the compiler would move them back and forth)
      }
      st[n].m = -INFINITY;
      st[n].shift = 0.f;
      st[n].l = 0.f;
    }
    __syncthreads();   // what was in the tiles has been read
    unsigned none = 0;   // two bits per granule, the latest requested lowest: its first, last 16 keys are on no page
    int page0, page1;
    auto next_pages = [&] {
      page0 = (unsigned)entry0 < (unsigned)p.n_pages ? entry0 : -1, page1 = (unsigned)entry1 < (unsigned)p.n_pages ? entry1 : -1;
      none = none << 2 | (page1 < 0) << 1 | (page0 < 0);
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; i++) {
      entry0 = entries[i][0], entry1 = entries[i][1];
      next_pages();
      if (AHEAD || g0 + i < g1) request(in_unit(g0 + i), i, page0, page1);
    }
    next_entries(in_unit(g0 + STAGES - 1));
    // The queries have been on their way with the first tiles.  (All are waited for here, once, and not by the first product in the loop.)
#pragma unroll
    for (int n = 0; n < R; n++) {
#pragma unroll
      for (int i = 0; i < STEPS; i++) asm volatile("" : "+v"(q[n][i]));
    }
    if (a.odd_scale) {
#pragma unroll
      for (int n = 0; n < R; n++) {
#pragma unroll
        for (int i = 0; i < STEPS; i++) q[n][i] = (q[n][i] ^ a.negate) & a.q_bits;
      }
    }

    int odd_from = g1;   // first granule with such values
    // A weight of zero does not silence an infinity or a NaN.  Committed values are seen by every row; where there is anything
    // that a row may not see, values that are no numbers are taken out of the tile here and given back, below, to the rows that see them.
    auto clean_values = [&](int granule, int stage, unsigned gone) {
      if ((granule + 1) * GRANULE <= length && gone == 0) return;
      unsigned char* const at = tiles[stage][1] + lane * 16;
      bool odd = false;
      for (int part = rw; part < PARTS; part += RW) odd |= clean<T, false>(at + part * 1024);
      if (__syncthreads_or(odd)) {
        odd_from = min(odd_from, granule);
        for (int part = rw; part < PARTS; part += RW) (void)clean<T, true>(at + part * 1024);
        __syncthreads();
      }
    };
    // The scores of a granule.  Reads of shared memory run LEAD steps in front of the products that take them (left to itself the
    // compiler puts a read right in front of its product, which then waits for the whole way there and back).  beside(i) goes
    // with the products of step i.  Of a result, 4 are of keys 4 quad .., 4 of those 16 further on.
    constexpr int LEAD = 3, LEAD_V = 4;
    auto scores = [&](int stage, f32x8 (&s)[R], auto beside) {
      const unsigned at = lds0 + stage * 2 * TILE;
      s16x8 kf[STEPS][2];
      f32x4 sum[R][2];
      auto read_keys = [&](int i) {
#pragma unroll
        for (int t = 0; t < 2; t++) kf[i][t] = *((LdsPiece)(size_t)(at + (read_k ^ ((4 * i & 12) << 4)) + t * 32 * D) + (4 * i & 16));
      };
#pragma unroll
      for (int i = 0; i < (LEAD < STEPS ? LEAD : STEPS); i++) read_keys(i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < STEPS; i++) {
        if (i + LEAD < STEPS) read_keys(i + LEAD);
#pragma unroll
        for (int n = 0; n < R; n++) {
#pragma unroll
          for (int t = 1; t >= 0; t--) sum[n][t] = Mat<T>::mfma(kf[i][t], q[n][i], i == 0 ? f32x4{} : sum[n][t]);   // (one wait for both)
        }
        beside(i);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int n = 0; n < R; n++) s[n] = __builtin_shufflevector(sum[n][0], sum[n][1], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    s16x8 vf[TILES];
    auto read_values = [&](int stage, int i) {   // of tile i
      const unsigned at = lds0 + stage * 2 * TILE + TILE + (read_v ^ ((i & 7) << 5)) + (i >> 3) * 256;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)(size_t)at);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)(size_t)(at + 32 * D));
      vf[i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto first_values = [&](int stage, int step) {   // those of the first LEAD_V tiles, with the last two steps of the scores
#pragma unroll
      for (int i = 0; i < LEAD_V / 2; i++) {
        if (step >= STEPS - 2) read_values(stage, (step - (STEPS - 2)) * (LEAD_V / 2) + i);
      }
    };
    // what of a tile the rows do not see becomes minus infinity.  gone: its first, last 16 keys are on no page
    auto hide = [&](f32x8 (&s)[R], int granule, unsigned gone) {
      const int pos0 = granule * GRANULE, j0 = pos0 - length;   // node at the tile's first key
      if (j0 + GRANULE <= 0 && gone == 0) return;
      unsigned on_page = 0xffffffffu;
      if (gone & 1) on_page &= 0xffff0000u;
      if (gone & 2) on_page &= 0x0000ffffu;
      const int have = total - pos0, committed = min(32, max(0, -j0)), jn = max(j0, 0);
      if (have < 32) on_page &= have > 0 ? (1u << have) - 1 : 0u;
#pragma unroll
      for (int n = 0; n < R; n++) {
        unsigned nodes = 0;             // bit b: node jn + b
        if (a.mask != nullptr) {
          const int word = jn >> 5, off = jn & 31;
          const unsigned lo = word < a.mask_words ? mask[n][word] : 0, hi = word + 1 < a.mask_words ? mask[n][word + 1] : 0;
          nodes = (unsigned)(((unsigned long long)hi << 32 | lo) >> off);
        } else {
          const int visible = node[n] - jn + 1;
          nodes = visible >= 32 ? 0xffffffffu : visible > 0 ? (1u << visible) - 1 : 0u;
        }
        // a bit per key
        const unsigned seen = on_page & (committed >= 32 ? 0xffffffffu : (1u << committed) - 1 | nodes << committed);
        const unsigned bits = seen >> (4 * quad);   // bit 16 (i / 4) + i % 4 is element i's key
#pragma unroll
        for (int i = 0; i < 8; i++) s[n][i] = bits >> (16 * (i >> 2) + (i & 3)) & 1 ? s[n][i] : -INFINITY;
      }
    };
    // The reference of the exponents is the maximum of a row's first granule, and follows it only where a weight would pass
    // 2^(8 + HEADROOM): hardly ever.  fp16 weights start at 2^HEADROOM, so that small ones keep their bits.  top: of this lane's scores
    constexpr float HEADROOM = Mat<T>::EXPONENT == 0x7c00 ? 7.f : 0.f;
    auto refer_to = [&](float (&top)[R]) {   // gives back in top what sums so far have to be multiplied by
#pragma unroll
      for (int n = 0; n < R; n++) {
        const float m = fmaxf(st[n].m, max_xor32(max_xor16(top[n])) * a.scale - HEADROOM);
        top[n] = st[n].m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[n].m - m);
        st[n].m = m;
        st[n].shift = m == -INFINITY ? 0.f : -m;
        st[n].l *= top[n];
      }
    };
    auto settle = [&](float (&top)[R]) {
      bool past = false, sums = false;
#pragma unroll
      for (int n = 0; n < R; n++) past |= top[n] * a.scale > st[n].m + (8.f + HEADROOM), sums |= st[n].m != -INFINITY;
      if (__ballot(past) != 0) {
        refer_to(top);
        if (__ballot(sums) != 0) {   // (not in the first granule: code that is not reached is not fetched)
#pragma unroll
          for (int n = 0; n < R; n++) scale_sums<TILES>(st[n].o, top[n]);
        }
      }
    };
    // Weights are rounded to the cache's type: the second product takes 16-bit operands, 32-bit ones have a sixteenth of the rate.  The
    // distance of results from 64 bits, norm over norm, is 2.3e-3 with it and 1.7e-3 by their own last rounding alone (8 x 64 nodes over 16384, bf16), 2.4e-4
    // and 2.1e-4 (16 x 33 over 3001, fp16).
    // (The empty assembly holds what is made beside products there: the compiler moves it behind the next branch otherwise.)
    unsigned pw[R][4];
    auto weigh = [&](const f32x8 (&s)[R], int pair) {   // two scores of this lane, of 4 R
      const int n = pair >> 2, i = pair & 3;
      T2 w;
      w[0] = (T)__builtin_amdgcn_exp2f(fmaf(s[n][2 * i], a.scale, st[n].shift));
      w[1] = (T)__builtin_amdgcn_exp2f(fmaf(s[n][2 * i + 1], a.scale, st[n].shift));
      st[n].l = dot_ones(w, st[n].l);   // of what the product takes, so that rounding a dominant weight cancels
      pw[n][i] = __builtin_bit_cast(unsigned, w);
      asm volatile("" : "+v"(pw[n][i]), "+v"(st[n].l));
    };
    auto sum_values = [&](int stage, auto beside) {
      s16x8 pf[R];
#pragma unroll
      for (int n = 0; n < R; n++) pf[n] = __builtin_bit_cast(s16x8, uint4{pw[n][0], pw[n][1], pw[n][2], pw[n][3]});
#pragma unroll
      for (int i = 0; i < TILES; i += 2) {
#pragma unroll
        for (int j = i + LEAD_V; j < i + LEAD_V + 2; j++) {
          if (j < TILES) read_values(stage, j);
        }
#pragma unroll
        for (int j = i + 1; j >= i; j--) {   // (one wait for both)
#pragma unroll
          for (int n = 0; n < R; n++) st[n].o[j] = Mat<T>::mfma(vf[j], pf[n], st[n].o[j]);
        }
        beside(i);
        beside(i + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // over scores from .. to - 1 of this lane's 8 R, which go from s to `to_s` (and out of the accumulation registers for good)
    auto maximum = [&](float (&top)[R], f32x8 (&to_s)[R], const f32x8 (&s)[R], int from, int to) {
#pragma unroll
      for (int i = 0; i < 8 * R; i += 2) {
        if (i < from || i >= to) continue;
        float a = s[i >> 3][i & 7], b = s[i >> 3][(i & 7) + 1];
        asm volatile("" : "+v"(a), "+v"(b));
        to_s[i >> 3][i & 7] = a, to_s[i >> 3][(i & 7) + 1] = b;
        top[i >> 3] = (i & 7) == 0 ? fmaxf(a, b) : fmaxf(top[i >> 3], fmaxf(a, b));
        asm volatile("" : "+v"(top[i >> 3]));
      }
    };
    // until a granule is there: AFTER granules behind it may be on their way, and all are waited for where the unit has fewer
    auto arrived = [&](int granule, auto after) {
      if (AHEAD || granule + after < g1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(after * REQUESTS) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();   // from every wave; and the granule before has been read by every wave
    };

    int stage = 0;
    if (row_tile * ROWS + rw * R * 16 >= rows.y * a.group) {
      // a wave without rows: its part of the requests, and what all waves do together
      if (AHEAD) arrived(g0, std::integral_constant<int, STAGES - 2>());
#pragma unroll 1
      for (int granule = g0; granule < g1; granule++) {
        arrived(granule + AHEAD, std::integral_constant<int, STAGES - 2 - AHEAD>());
        clean_values(granule, stage, none >> (2 * (STAGES - 2)) & 3);
        const int wanted = granule + STAGES - 1;
        next_pages();
        if (AHEAD || wanted < g1) request(in_unit(wanted), stage == 0 ? STAGES - 1 : stage - 1, page0, page1);
        next_entries(in_unit(wanted + 1));
        stage = stage + 1 == STAGES ? 0 : stage + 1;
      }
    } else if constexpr (AHEAD) {
      // scores one granule ahead: their products run beside the exponentials of the granule whose values are summed next
      arrived(g0, std::integral_constant<int, STAGES - 2>());
      f32x8 s[R], s_next[R];
      float top[R];
      scores(0, s, [](int) {});
      hide(s, g0, none >> (2 * (STAGES - 2)) & 3);
      maximum(top, s, s, 0, 8 * R);
      refer_to(top);
#pragma unroll 1
      for (int granule = g0; granule < g1; granule++) {
        arrived(granule + 1, std::integral_constant<int, STAGES - 3>());
        clean_values(granule, stage, none >> (2 * (STAGES - 2)) & 3);
        const int stage1 = stage + 1 == STAGES ? 0 : stage + 1, wanted = granule + STAGES - 1;
        next_pages();
        const Quarter at = quarter_of(in_unit(wanted), stage == 0 ? STAGES - 1 : stage - 1, page0, page1);
        scores(stage1, s_next, [&](int i) {
          first_values(stage, i);
#pragma unroll
          for (int j = i * (QUARTER / BURST) / STEPS; j < (i + 1) * (QUARTER / BURST) / STEPS; j++) request_burst(at, j);
#pragma unroll
          for (int j = i * 4 * R / STEPS; j < (i + 1) * 4 * R / STEPS; j++) weigh(s, j);
        });
        if (granule + 1 < g1) hide(s_next, granule + 1, none >> (2 * (STAGES - 2)) & 3);
        sum_values(stage, [&](int i) { maximum(top, s, s_next, i * 8 * R / TILES, (i + 1) * 8 * R / TILES); });
        next_entries(in_unit(wanted + 1));
        if (granule + 1 < g1) settle(top);
        stage = stage1;
      }
    } else {
      f32x8 s[R];
      float top[R];
      for (int granule = g0; granule < g1; granule++) {
        arrived(granule, std::integral_constant<int, STAGES - 2>());
        clean_values(granule, stage, none >> (2 * (STAGES - 2)) & 3);
        const int wanted = granule + STAGES - 1;
        next_pages();
        if (wanted < g1) request(wanted, stage == 0 ? STAGES - 1 : stage - 1, page0, page1);
        scores(stage, s, [&](int i) { first_values(stage, i); });
        hide(s, granule, none >> (2 * (STAGES - 1)) & 3);
        maximum(top, s, s, 0, 8 * R);
        settle(top);
#pragma unroll
        for (int j = 0; j < 4 * R; j++) weigh(s, j);
        sum_values(stage, [](int) {});
        next_entries(in_unit(wanted + 1));
        stage = stage + 1 == STAGES ? 0 : stage + 1;
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing is on its way to the tiles any more
#pragma unroll
    for (int n = 0; n < R; n++) {
      RowState<D>& row = st[n];
      row.l = add_xor32(add_xor16(row.l));
      if (!live[n]) continue;
      if (odd_from < g1) {
        // rare: sums that such values are part of are what adding them makes of any number
#pragma unroll 1
        for (int pos = odd_from * GRANULE; pos < min(total, g1 * GRANULE); pos++) {
          const int j = pos - length, page = page_at(p, seq, pos >> shift);
          const bool sees = j < 0 || (a.mask != nullptr ? (j >> 5) < a.mask_words && (mask[n][j >> 5] >> (j & 31) & 1) : j <= node[n]);
          if (!sees || page < 0) continue;
          const T* v_row = reinterpret_cast<const T*>(pool_v) + page * p.page_stride + (pos & in_page) * p.token_stride + 4 * quad;
#pragma unroll
          for (int b = 0; b < TILES; b++) {
            const T4 v = *reinterpret_cast<const T4*>(v_row + b * 16);
#pragma unroll
            for (int i = 0; i < 4; i++) {
              const float x = (float)v[i];
              row.o[b][i] += x - x == 0.f ? 0.f : x;
            }
          }
        }
      }
      if (g0 == 0 && g1 == granules) {
        const float inv = row.l == 0.f ? 0.f : 1.0f / row.l;
        T* out = reinterpret_cast<T*>(a.out) + (rows.x + node[n]) * a.out_row_stride + head[n] * a.out_head_stride;
#pragma unroll
        for (int b = 0; b < TILES; b++) {
          T4 w;
#pragma unroll
          for (int i = 0; i < 4; i++) w[i] = (T)(row.o[b][i] * inv);
          *reinterpret_cast<T4*>(out + b * 16 + 4 * quad) = w;
        }
      } else {
        const size_t set = ((size_t)blockIdx.x * 2 + (g0 == 0)) * a.sets + rw * R + n;
#pragma unroll
        for (int b = 0; b < TILES; b++) a.part_o[(set * TILES + b) * 64 + lane] = row.o[b];
        if (quad == 0) a.part_ml[set * 16 + kkey] = make_float2(row.m, row.l);
      }
    }
  }
}

// The rows of units that several blocks had a part in: sum_z 2^(m_z - m) o_z / sum_z 2^(m_z - m) l_z, in the order of the keys.  A wave
// has 16 d of 16 rows, as the partial results lie; WPR waves share out the parts: 8 where units are so few that each has many, with both
// launches 8 and 1 of 1 token over 16384 12.2 and 30.2 us, of 4 x 8 over 4096 13.9 and 18.0, of 16 x 33 over 4096 51.2 and 44.6.  Bound
// by the partial results, 64 KiB R per block of heads of 256 and twice that where a run ends one unit and begins another.
template <class T, int D, int R, int WPR>
__global__ __launch_bounds__(512) void tree_merge_kernel(TreeArgs a) {
  constexpr int ROWS = 16 * R * RW, TILES = D / 16, BATCH = 4;
  typedef T T4 __attribute__((ext_vector_type(4)));
  const pi0_pages& p = a.p;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nth = wave % WPR, kkey = lane & 15, quad = lane >> 4;
  const int item = blockIdx.x * (8 / WPR) + wave / WPR, set = item / TILES, tile = item % TILES, kv_head = blockIdx.y, seq = blockIdx.z;
  const int2 rows = rows_of(a.row_start, seq, a.n_rows, a.max_rows);
  if (set * 16 >= rows.y * a.group) return;   // (with WPR == 8 all of a block's waves)
  const int total = min(length_of(p, seq) + rows.y, p.max_pages * p.page_tokens);
  const int granules = div_up(total, GRANULE), row_tiles = div_up(rows.y * a.group, ROWS), row_tile = set / (ROWS / 16);
  const int run = *a.run, share = granules + START;
  const int first = (seq > 0 ? a.upto[seq - 1] : 0) + (kv_head * row_tiles + row_tile) * share + START;
  const int run0 = first / run, parts = (first + granules - 1) / run - run0 + 1;   // the runs that had a part
  if (parts < 2) return;
  // this wave's parts, each row against the maximum of its own so far; what a row that is not there holds stays in its lanes
  f32x4 o = {};
  float m = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int part = nth; part < parts; part += BATCH * WPR) {
    float2 ml[BATCH];
    f32x4 v[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; i++) {
      const int z = part + i * WPR;
      const size_t from = ((size_t)(run0 + min(z, parts - 1)) * 2 + (z == 0)) * a.sets + set % (ROWS / 16);
      ml[i] = a.part_ml[from * 16 + kkey];
      v[i] = a.part_o[(from * TILES + tile) * 64 + lane];
      if (z >= parts) ml[i].x = -INFINITY, v[i] = f32x4{};
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < BATCH; i++) top = fmaxf(top, ml[i].x);
    const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
    o *= keep, l *= keep, m = top;
#pragma unroll
    for (int i = 0; i < BATCH; i++) {
      const float c = ml[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[i].x - m);
      o += c * v[i], l += c * ml[i].y;
    }
  }
  if constexpr (WPR > 1) {
    __shared__ float2 s_ml[WPR][16];
    __shared__ f32x4 s_o[WPR][64];
    if (quad == 0) s_ml[nth][kkey] = make_float2(m, l);
    s_o[nth][lane] = o;
    __syncthreads();
    if (nth != 0) return;
    for (int w = 1; w < WPR; w++) m = fmaxf(m, s_ml[w][kkey].x);
    o = f32x4{}, l = 0.f;
    for (int w = 0; w < WPR; w++) {
      const float2 ml = s_ml[w][kkey];
      const float c = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
      o += c * s_o[w][lane], l += c * ml.y;
    }
  }
  const int r = set * 16 + kkey;
  if (r >= rows.y * a.group) return;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const int node = r / a.group, head = kv_head * a.group + r - node * a.group;
  T4 w;
#pragma unroll
  for (int i = 0; i < 4; i++) w[i] = (T)(o[i] * inv);
  *reinterpret_cast<T4*>(reinterpret_cast<T*>(a.out) + (rows.x + node) * a.out_row_stride + head * a.out_head_stride + tile * 16 + 4 * quad) = w;
}

struct Space {
  int sets;
  size_t part_ml, upto, run, bytes;   // part_o lies in front
};
template <int D, int R>
Space space_of(const pi0_pages& p, int rows) {
  Space s;
  s.sets = min(4 * R, div_up(rows, 16));
  const size_t slots = (size_t)Shape<D, R>::BLOCKS * 2 * 16 * s.sets;
  s.part_ml = slots * D * sizeof(float);
  s.upto = s.part_ml + slots * sizeof(float2);
  s.run = s.upto + (size_t)p.n_seqs * sizeof(int);
  s.bytes = s.run + sizeof(int);
  return s;
}

// f(R): 64 rows per tile, or 128 where there are more than that of enough sequences and heads (measured with 64 and with 128: 8 x 64 nodes
// with 8 heads over 1 of 256 and 16384 keys 61.8 and 57.3 us, 16 x 33 with 32 over 8 of 128 and 4096 51.5 and 44.8; 1 x 64 over 2048
// 20.8 and 23.4, 16 x 16, that is 128 rows, over 2048 20.2 and 23.3).  192 rows per tile fit the registers of heads of 256 (242 + 228) and are as fast
// for 8 x 64, and spill for heads of 128.
template <class F>
auto with_rows(int rows, int heads, F f) {
  if (rows > 128 && heads >= 4) return f(std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 1>());
}
template <class F>
auto with_dim(int head_dim, F f) {
  if (head_dim == 64) return f(std::integral_constant<int, 64>());
  if (head_dim == 128) return f(std::integral_constant<int, 128>());
  return f(std::integral_constant<int, 256>());
}

Space space_of(const pi0_pages& p, int heads, int max_rows) {
  const int rows = max_rows * (heads / p.kv_heads);
  return with_dim(p.head_dim, [&](auto d) {
    return with_rows(rows, p.n_seqs * p.kv_heads, [&](auto r) { return space_of<d, r>(p, rows); });
  });
}

template <class T>
hipError_t launch(hipStream_t s, TreeArgs& a, char* ws) {
  return with_dim(a.p.head_dim, [&](auto d) {
    const int rows = a.max_rows * a.group;
    return with_rows(rows, a.p.n_seqs * a.p.kv_heads, [&](auto r) {
      constexpr int D = d, R = r, BLOCKS = Shape<D, R>::BLOCKS;
      const Space at = space_of<D, R>(a.p, rows);
      a.sets = at.sets;
      a.part_o = reinterpret_cast<f32x4*>(ws);
      a.part_ml = reinterpret_cast<float2*>(ws + at.part_ml);
      a.upto = reinterpret_cast<int*>(ws + at.upto);
      a.run = reinterpret_cast<int*>(ws + at.run);
      const hipError_t e = enqueue(s, dim3(BLOCKS), 64 * RW, tree_attention_kernel<T, D, R>, a);
      if (e != hipSuccess) return e;
      const int units = a.p.n_seqs * a.p.kv_heads * div_up(rows, 16 * R * RW);
      const int items = div_up(rows, 16) * (D / 16);   // of 16 rows and 16 d
      if (units <= BLOCKS / 16)
        return enqueue(s, dim3(items, a.p.kv_heads, a.p.n_seqs), 512, tree_merge_kernel<T, D, R, 8>, a);
      return enqueue(s, dim3(div_up(items, 8), a.p.kv_heads, a.p.n_seqs), 512, tree_merge_kernel<T, D, R, 1>, a);
    });
  });
}

bool args_ok(const pi0_pages* p, int heads, int n_rows, int max_rows) {
  if (!pages_ok(p) || heads < 1 || heads > 1024 || heads % p->kv_heads != 0) return false;
  if (n_rows < 1 || n_rows > 1 << 24 || max_rows < 1 || max_rows > 1024 || max_rows > n_rows) return false;
  // the line of all units' granules is counted in 31 bits
  const int64_t tiles = div_up(max_rows * (heads / p->kv_heads), 16), granules = div_up(p->max_pages * p->page_tokens, GRANULE) + START;
  return (int64_t)p->n_seqs * p->kv_heads * tiles * granules < (int64_t)1 << 30;
}

}  // namespace

extern "C" {

size_t pi0_tree_attention_workspace_bytes(const pi0_pages* pages, int heads, int n_rows, int max_rows) {
  return args_ok(pages, heads, n_rows, max_rows) ? space_of(*pages, heads, max_rows).bytes : 0;
}

int pi0_tree_attention(const pi0_pages* pages, int layer, const pi0_rows* q, const pi0_rows* out, const int32_t* d_row_start, int n_rows,
                       int max_rows, const uint32_t* d_mask, int mask_words, float scale, void* d_workspace, size_t ws_bytes, void* hip_stream) {
  if (q == nullptr || d_row_start == nullptr || ((uintptr_t)d_row_start & 3) != 0 || !args_ok(pages, q->heads, n_rows, max_rows)) return PI0_EINVAL;
  if (layer < 0 || layer >= pages->layers || !(fabsf(scale) < 0x1p127f)) return PI0_EINVAL;   // (times log2(e) it is still a number)
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
  a.group = q->heads / pages->kv_heads;
  a.row_start = d_row_start;
  a.n_rows = n_rows;
  a.max_rows = max_rows;
  a.mask = d_mask;
  a.mask_words = mask_words;
  a.scale = fabsf(scale) * 1.4426950408889634f;
  a.odd_scale = !(scale > 0.f);
  a.negate = scale < 0.f ? (short)0x8000 : 0;
  a.q_bits = -1;
  if (a.scale == 0.f) {   // all scores are zero, and a masked one stays minus infinity
    a.q_bits = 0;
    a.scale = 1.f;
  }
  a.layer = layer * pages->layer_stride;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  char* const ws = reinterpret_cast<char*>(d_workspace);
  const hipError_t e = pages->dtype == PI0_BF16 ? launch<bf16>(s, a, ws) : launch<f16>(s, a, ws);
  return e == hipSuccess ? PI0_OK : PI0_EHIP;
}

}  // extern "C"
