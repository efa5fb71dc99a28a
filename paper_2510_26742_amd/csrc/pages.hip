// Page operations of a paged key/value cache: reserve, fork, compact; the way between pages and a ctx's cache.
//
// Every operation that changes a table is planned by one block of 1024 threads - a wave per sequence, prefix sums over
// sequences and over free pages - and, where rows move, carried out by a second launch over (sequence, layer, key /
// value).  The plan is written only after everything it checks has been found right, so a refused call changes nothing,
// and whatever it decides by (reference counts, free pages) is read before any of it is written: neither the order of
// the waves nor that of the sequences changes what comes out, but for the ascending order in which free pages go to
// ascending sequences.  Pages that a call releases are handed out by the next call at the earliest, so the rows of the
// second launch are read from pages that nobody writes.
#include "pages_common.h"

#include <string.h>

bool pages_ok(const pi0_pages* p) {
  if (p == nullptr || p->d_k == nullptr || p->d_v == nullptr || p->d_table == nullptr || p->d_length == nullptr || p->d_refs == nullptr ||
      p->d_status == nullptr)
    return false;
  if (((uintptr_t)p->d_k | (uintptr_t)p->d_v) & 15) return false;
  if (((uintptr_t)p->d_table | (uintptr_t)p->d_length | (uintptr_t)p->d_refs | (uintptr_t)p->d_status) & 3) return false;
  if (p->dtype != PI0_BF16 && p->dtype != PI0_F16) return false;
  if (p->layers < 1 || p->layers > 1 << 16 || p->n_pages < 1 || p->n_pages > 1 << 24) return false;
  if (p->page_tokens < 16 || p->page_tokens > 256 || (p->page_tokens & (p->page_tokens - 1)) != 0) return false;
  if (p->kv_heads < 1 || p->kv_heads > 256) return false;
  if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256) return false;
  if (p->n_seqs < 1 || p->n_seqs > MAX_SEQS || p->max_pages < 1 || (int64_t)p->max_pages * p->page_tokens > 1 << 24) return false;
  // (the moves' grid, a block of 256 threads per 128 elements of a layer, has less than 2^32 threads)
  if ((int64_t)p->layers * p->kv_heads * p->head_dim > 1 << 29) return false;
  if (p->token_stride >= (int64_t)1 << 27) return false;
  // strides: whole 16-byte pieces, and, from the innermost axis outwards, each axis beyond all that lies inside it
  int64_t stride[4] = {p->layer_stride, p->page_stride, p->token_stride, p->head_stride};
  int64_t count[4] = {p->layers, p->n_pages, p->page_tokens, p->kv_heads};
  int64_t inside = p->head_dim;
  for (int done = 0; done < 4; done++) {
    int at = done;
    for (int i = done + 1; i < 4; i++) {
      if (stride[i] < stride[at]) at = i;
    }
    const int64_t s = stride[at], c = count[at];
    stride[at] = stride[done], count[at] = count[done];
    if (s < 0 || s % 8 != 0 || s > (int64_t)1 << 46) return false;
    if (c == 1) continue;
    if (s < inside) return false;
    inside = s * (c - 1) + inside;
    if (inside > (int64_t)1 << 46) return false;
  }
  return true;
}

bool rows_ok(const pi0_rows* r, int heads, int head_dim, int dtype) {
  if (r == nullptr || r->d_x == nullptr || ((uintptr_t)r->d_x & 15) != 0 || r->dtype != dtype) return false;
  if (r->heads < 1 || r->heads > 1024 || (heads != 0 && r->heads != heads)) return false;
  if (r->row_stride < head_dim || r->row_stride % 8 != 0 || r->row_stride > (int64_t)1 << 40) return false;
  return r->head_stride >= head_dim && r->head_stride % 8 == 0 && r->head_stride <= (int64_t)1 << 40;
}

namespace {

constexpr int PLAN_THREADS = 1024, PLAN_WAVES = PLAN_THREADS / 64;

// what the second launch does for a sequence: positions [begin, end) of its new list come from `from + keep[pos - from]`
// (pos < from: from the same position) of the list as it was before
struct Move {
  int begin, end, from;
  int held;   // pages of the list as it was
};
// workspace: moves [n_seqs], the lists as they were [n_seqs][max_pages], the free pages that are handed out [n_pages]
constexpr int SHARED = 1 << 30;   // in an entry of a list as it was: others hold the page too, and it is replaced
struct PlanSpace {
  Move* moves;
  int* before;
  int* free_pages;
};
size_t plan_bytes(const pi0_pages& p) {
  return round_up_sz(sizeof(Move) * p.n_seqs, 16) + round_up_sz(4 * (size_t)p.n_seqs * p.max_pages, 16) + 4 * (size_t)p.n_pages;
}
PlanSpace plan_space(const pi0_pages& p, void* ws) {
  char* at = reinterpret_cast<char*>(ws);
  PlanSpace s;
  s.moves = reinterpret_cast<Move*>(at);
  at += round_up_sz(sizeof(Move) * p.n_seqs, 16);
  s.before = reinterpret_cast<int*>(at);
  at += round_up_sz(4 * (size_t)p.n_seqs * p.max_pages, 16);
  s.free_pages = reinterpret_cast<int*>(at);
  return s;
}

__device__ __forceinline__ int wave_min(int v) {
  for (int i = 32; i > 0; i >>= 1) v = min(v, __shfl_xor(v, i));
  return v;
}
__device__ __forceinline__ int wave_sum(int v) {
  for (int i = 32; i > 0; i >>= 1) v += __shfl_xor(v, i);
  return v;
}
__device__ __forceinline__ int lanes_below(unsigned long long mask) {
  return __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
}

// pages in front of a sequence's list (by a whole wave, each lane of which has read its entry of the first 64)
__device__ int pages_held(const pi0_pages& p, int seq, int lane, int entry) {
  for (int at = 0;; entry = page_at(p, seq, at + lane)) {
    const unsigned long long none = __ballot(entry < 0);
    if (none != 0) return min(p.max_pages, at + __ffsll(none) - 1);
    at += 64;
    if (at >= p.max_pages) return p.max_pages;
  }
}

// exclusive prefix sum of `mine` over the block's threads; *total gets the sum.  sums: PLAN_WAVES ints of shared memory
__device__ int block_prefix(int mine, int* sums, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int v = mine;
  for (int i = 1; i < 64; i <<= 1) {
    const int u = __shfl_up(v, i);
    if (lane >= i) v += u;
  }
  __syncthreads();   // the sums of a call before have been read
  if (lane == 63) sums[wave] = v;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < PLAN_WAVES; w++) {
    if (w < wave) before += sums[w];
    all += sums[w];
  }
  *total = all;
  return before + v - mine;
}

// What a plan went by is read again when it is carried out, from memory that is the caller's.  Were it changed meanwhile, the
// cache would be wrong; but no address is formed from a number that has not just been checked.
__device__ __forceinline__ void take(const pi0_pages& p, int* entry, int page) {
  if ((unsigned)page >= (unsigned)p.n_pages) return;
  *entry = page;
  p.d_refs[page] = 1;
}
__device__ __forceinline__ void release(const pi0_pages& p, int page) {
  if ((unsigned)page < (unsigned)p.n_pages) atomicSub(&p.d_refs[page], 1);
}

enum PlanKind { PLAN_RESERVE, PLAN_COMPACT };
struct PlanArgs {
  pi0_pages p;
  PlanSpace ws;
  const int* extra;     // reserve
  const int* start;     // compact
  const int* keep;
  const int* n_keep;
  int keep_stride;
};

// For every sequence that takes part:  [first, last) of its list may hold pages that others hold too and that rows are written
// to - those are replaced -, the list has `want` pages afterwards, of which it holds `held` now.  reserve: want >= held,
// compact: want <= held.  What bounds it is trips to memory (0.6 us each) and 16 waves for all sequences, so: numbers
// that all sequences have are read at once, a list and the positions that it keeps in one trip, reference counts in a second, and what
// was found is left in the workspace for the second half (4 sequences 5.8 us for a compaction and 4.6 for a reservation, 48 with 560 positions each
// 12.9 and 7.8).  The free pages cost one trip per 1024 reference counts until enough are found.
template <int KIND>
__global__ __launch_bounds__(PLAN_THREADS) void pages_plan_kernel(PlanArgs a) {
  const pi0_pages& p = a.p;
  __shared__ int s_need[MAX_SEQS], s_first[MAX_SEQS], s_last[MAX_SEQS], s_held[MAX_SEQS], s_want[MAX_SEQS], s_length[MAX_SEQS], s_n[MAX_SEQS];
  __shared__ int s_sums[PLAN_WAVES], s_bad;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  if (t == 0) s_bad = 0;
  if (t < p.n_seqs) {
    s_n[t] = KIND == PLAN_RESERVE ? a.extra[t] : a.n_keep[t];
    s_length[t] = p.d_length[t];
    s_first[t] = KIND == PLAN_COMPACT && a.start != nullptr ? a.start[t] : s_length[t];
  }
  __syncthreads();
  for (int s = wave; s < p.n_seqs; s += PLAN_WAVES) {
    const int n = s_n[s], length = s_length[s];
    int need = 0, first = 0, last = 0, held = 0, want = -1;   // want < 0: the sequence stays as it is
    Move m = {0, 0, 0, 0};
    if (n >= 0) {
      const int entry = page_at(p, s, lane);
      bool bad = length < 0;
      if (KIND == PLAN_RESERVE) {
        held = pages_held(p, s, lane, entry);
        bad |= length > held * p.page_tokens || (int64_t)length + n > (int64_t)p.max_pages * p.page_tokens;
        if (!bad) {
          want = max(held, div_up(length + n, p.page_tokens));
          first = length / p.page_tokens;
          last = n > 0 ? min(held, div_up(length + n, p.page_tokens)) : first;
          m = {first * p.page_tokens, length, length, held};   // the committed rows of the first replaced page, if it is replaced
        }
      } else {
        const int start = s_first[s];
        bad |= n > a.keep_stride || start < 0 || start > length;
        int moved = n, furthest = -1;
        if (!bad) {
          constexpr int DEEP = 8;   // in flight
          const int* keep = a.keep + (size_t)s * a.keep_stride;
          for (int at = lane; at < n; at += 64 * DEEP) {
            int k[DEEP], in_front[DEEP];
#pragma unroll
            for (int j = 0; j < DEEP; j++) k[j] = keep[min(at + 64 * j, n - 1)], in_front[j] = keep[max(min(at + 64 * j, n - 1) - 1, 0)];
#pragma unroll
            for (int j = 0; j < DEEP; j++) {
              const int i = min(at + 64 * j, n - 1);
              bad |= k[j] < 0 || (i > 0 && k[j] <= in_front[j]);
              if (k[j] != i) moved = min(moved, i);
              furthest = max(furthest, k[j]);
            }
          }
        }
        held = pages_held(p, s, lane, entry);
        bad |= length > held * p.page_tokens || (furthest >= 0 && (int64_t)start + furthest >= (int64_t)held * p.page_tokens);
        bad = __ballot(bad) != 0;
        moved = wave_min(moved);
        if (!bad) {
          const int begin = start + moved, end = start + n;
          want = div_up(end, p.page_tokens);
          first = begin / p.page_tokens;
          last = begin < end ? want : first;
          m = {begin, end, start, held};
        }
      }
      if (bad) {
        s_bad = 1;
      } else {
        int* before = a.ws.before + (size_t)s * p.max_pages;
        for (int i = lane; i < held; i += 64) {
          const int page = i < 64 ? entry : page_at(p, s, i);
          const bool shared = i >= first && i < last && p.d_refs[max(page, 0)] > 1;
          before[i] = shared ? page | SHARED : page;
          need += shared;
        }
        need = wave_sum(need) + max(0, want - held);
      }
    }
    if (lane == 0) {
      s_need[s] = need, s_first[s] = first, s_last[s] = last, s_held[s] = held, s_want[s] = want;
      a.ws.moves[s] = m;
    }
  }
  __syncthreads();
  bool bad = s_bad != 0;
  int total = 0;
  const int base = block_prefix(t < p.n_seqs ? s_need[t] : 0, s_sums, &total);
  int found = 0;
  for (int at = 0; !bad && found < total && at < p.n_pages; at += PLAN_THREADS) {
    const bool is_free = at + t < p.n_pages && p.d_refs[at + t] == 0;
    int here = 0;
    const int rank = found + block_prefix(is_free, s_sums, &here);
    if (is_free && rank < total) a.ws.free_pages[rank] = at + t;
    found += here;
  }
  if (bad || found < total) {
    if (t == 0) *p.d_status = bad ? PI0_EINVAL : PI0_ENOMEM;
    for (int s = t; s < p.n_seqs; s += PLAN_THREADS) a.ws.moves[s] = {0, 0, 0, 0};
    return;
  }
  if (t < p.n_seqs) s_need[t] = base;   // from here on: the sequence's place among the free pages
  __syncthreads();
  // lists and reference counts
  auto handed_out = [&](int rank) { return rank < total ? a.ws.free_pages[rank] : -1; };
  for (int s = wave; s < p.n_seqs; s += PLAN_WAVES) {
    const int want = s_want[s], held = s_held[s], first = s_first[s], last = s_last[s];
    if (want < 0) continue;
    int* list = p.d_table + (size_t)s * p.max_pages;
    const int* before = a.ws.before + (size_t)s * p.max_pages;
    int next = s_need[s];
    bool first_replaced = false;
    for (int at = first; at < last; at += 64) {
      const int i = at + lane, entry = i < last ? before[i] : 0;
      const bool shared = (entry & SHARED) != 0;
      const unsigned long long mask = __ballot(shared);
      if (shared) {
        take(p, list + i, handed_out(next + lanes_below(mask)));
        release(p, entry & ~SHARED);
      }
      if (at == first) first_replaced = (mask & 1) != 0;
      next += __popcll(mask);
    }
    for (int i = held + lane; i < want; i += 64) take(p, list + i, handed_out(next + i - held));
    for (int i = want + lane; i < held; i += 64) {   // what the list no longer holds
      release(p, before[i]);
      list[i] = -1;
    }
    if (lane == 0) {
      Move m = a.ws.moves[s];
      if (KIND == PLAN_RESERVE) {
        if (!first_replaced) a.ws.moves[s] = {0, 0, 0, 0};
      } else {
        // a page of its own in front: the rows that stay where they are come with it
        if (first_replaced) a.ws.moves[s].begin = first * p.page_tokens;
        p.d_length[s] = m.end;
      }
    }
  }
}

// The rows of a plan.  A block moves 256 bytes of each of one sequence's rows of one layer of the keys or of the values:
// 16 threads of 16 bytes per row, 16 rows side by side, MOVE_ROWS deep.  In place a row only ever moves down, and
// ascending sources go to ascending places: the place of a row is no source of a row behind it, so loads may run ahead
// of stores, and a block-wide wait between the loads of a round and its stores keeps a store from overtaking the load
// of the row that it replaces.  Bound by memory and by the longest sequence's blocks: 32 continuations of 16 prefixes, 6100 rows of 512 bytes
// of 18 layers, 225 MB, in 85 us with the two plans and the fork around it; with 512 bytes per block and 8 rows deep 105, with 8 rows of
// 256 bytes 88, with 4 rows of 128 bytes 85, with 2 86.
constexpr int MOVE_ROWS = 4, MOVE_PIECES = 16;
__global__ __launch_bounds__(256) void pages_move_kernel(pi0_pages p, PlanSpace ws, const int* keep_all, int keep_stride) {
  const int s = blockIdx.y;
  const Move m = ws.moves[s];
  if (m.begin >= m.end) return;
  const int pieces = p.kv_heads * p.head_dim / 8, groups = div_up(pieces, MOVE_PIECES);
  const int group = blockIdx.x % groups, layer = blockIdx.x / groups >> 1;
  char* pool = reinterpret_cast<char*>((blockIdx.x / groups & 1) ? p.d_v : p.d_k) + 2 * layer * p.layer_stride;
  const int wide = min(MOVE_PIECES, pieces - group * MOVE_PIECES), deep = 256 / wide;
  const int row = threadIdx.x / wide, piece = group * MOVE_PIECES + threadIdx.x % wide;
  const int per_head = p.head_dim / 8;
  pool += 2 * ((piece / per_head) * p.head_stride + (piece % per_head) * 8);
  const int* now = p.d_table + (size_t)s * p.max_pages;
  const int* before = ws.before + (size_t)s * p.max_pages;
  const int* keep = keep_all + (size_t)s * keep_stride;
  const int shift = 31 - __clz(p.page_tokens), mask = p.page_tokens - 1;
  for (int at = m.begin; at < m.end; at += MOVE_ROWS * deep) {
    uint4 data[MOVE_ROWS];
    int64_t dst[MOVE_ROWS];
#pragma unroll
    for (int u = 0; u < MOVE_ROWS; u++) {
      const int pos = at + u * deep + row;
      dst[u] = -1;
      data[u] = uint4{};
      if (row < deep && pos < m.end) {
        const int src = pos < m.from ? pos : m.from + keep[pos - m.from];
        const int to = now[pos >> shift], from = src >= 0 && (src >> shift) < m.held ? before[src >> shift] & ~SHARED : -1;
        if ((unsigned)to < (unsigned)p.n_pages && (unsigned)from < (unsigned)p.n_pages) {
          dst[u] = 2 * (to * p.page_stride + (pos & mask) * p.token_stride);
          data[u] = *reinterpret_cast<const uint4*>(pool + 2 * (from * p.page_stride + (src & mask) * p.token_stride));
        }
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int u = 0; u < MOVE_ROWS; u++) {
      if (dst[u] >= 0) *reinterpret_cast<uint4*>(pool + dst[u]) = data[u];
    }
  }
}

// A wave per pair, everything checked before anything is written.  Bound by four trips to memory: 2.9 us for 3 continuations, 5.0 for 32.
__global__ __launch_bounds__(PLAN_THREADS) void pages_fork_kernel(pi0_pages p, const int* src, const int* dst, int n) {
  __shared__ int s_mark[MAX_SEQS], s_src[MAX_SEQS], s_dst[MAX_SEQS], s_bad;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  s_mark[t] = 0;
  if (t < n) s_src[t] = src[t], s_dst[t] = dst[t];
  if (t == 0) s_bad = 0;
  __syncthreads();
  for (int i = wave; i < n; i += PLAN_WAVES) {
    const int s = s_src[i];
    if (s < 0 || s >= p.n_seqs) {
      s_bad = 1;
      continue;
    }
    const int length = p.d_length[s];
    if (length < 0 || length > pages_held(p, s, lane, page_at(p, s, lane)) * p.page_tokens) s_bad = 1;
    if (lane == 0) atomicOr(&s_mark[s], 1);
  }
  __syncthreads();
  if (t < n) {
    const int d = s_dst[t];
    if (d < 0 || d >= p.n_seqs || atomicOr(&s_mark[d], 2) != 0) s_bad = 1;
  }
  __syncthreads();
  if (s_bad) {
    if (t == 0) *p.d_status = PI0_EINVAL;
    return;
  }
  for (int i = wave; i < n; i += PLAN_WAVES) {
    const int s = s_src[i], d = s_dst[i], length = length_of(p, s), shared = div_up(length, p.page_tokens);
    const int held = pages_held(p, d, lane, page_at(p, d, lane));
    int* list = p.d_table + (size_t)d * p.max_pages;
    for (int j = lane; j < max(shared, held); j += 64) {
      const int old = j < held ? list[j] : -1, page = j < shared ? page_at(p, s, j) : -1;
      if (old >= 0) release(p, old);
      if (page >= 0) atomicAdd(&p.d_refs[page], 1);
      list[j] = page;
    }
    if (lane == 0) p.d_length[d] = length;
  }
}

// Whether sequence seq holds pages of its own for `tokens` positions (by every thread of a block; tokens <= 1024, so at
// most 64 pages: one wave's lanes).  0, or the code to report.
__device__ int own_pages(const pi0_pages& p, int seq, int tokens) {
  const int lane = threadIdx.x & 63, n = div_up(tokens, p.page_tokens);
  const int page = lane < n ? page_at(p, seq, lane) : -1;
  if (__ballot(lane < n && page < 0) != 0) return PI0_ENOMEM;
  return __ballot(lane < n && p.d_refs[max(page, 0)] != 1) != 0 ? PI0_EINVAL : 0;
}

// One block: 32 tokens of one layer between the fragment order that the attention kernels of the pass read (32 keys x 256 per
// 16 KiB chunk; values transposed) and rows of pages.  Rows are 512 bytes, fragments 16-byte pieces of one key or, of the
// values, of 8 keys at one d: those pass through shared memory.  Bound by memory and the way there: 816 tokens of 18 layers, 30 MB read and
// written, 9.0 us to pages and 7.5 us back.
constexpr int CHUNK = 32, VROW = 256 + 8;
__device__ __forceinline__ bf16* page_row(const pi0_pages& p, void* pool, int layer, int seq, int pos) {
  const int page = page_at(p, seq, pos / p.page_tokens);
  if (page < 0) return nullptr;
  return reinterpret_cast<bf16*>(pool) + layer * p.layer_stride + page * p.page_stride + (pos % p.page_tokens) * p.token_stride;
}
// of value fragment piece i (0 .. 1023): its d, and the key of its element j
__device__ __forceinline__ int vfrag_d(int i) { return (i >> 7) * 32 + (i & 31); }
__device__ __forceinline__ int vfrag_key(int i, int j) { return ((i >> 6) & 1) * 16 + (j >> 2) * 8 + ((i >> 5) & 1) * 4 + (j & 3); }

__global__ __launch_bounds__(256) void pages_store_kernel(pi0_pages p, int seq, const bf16* kc, const bf16* vc, size_t k_layer, size_t v_layer, int tokens) {
  const int code = own_pages(p, seq, tokens), t = threadIdx.x, chunk = blockIdx.x, layer = blockIdx.y;
  if (code != 0) {
    if (chunk == 0 && layer == 0 && t == 0) *p.d_status = code;
    return;
  }
  const bf16x8* kf = reinterpret_cast<const bf16x8*>(reinterpret_cast<const char*>(kc) + layer * k_layer) + (size_t)chunk * 1024;
  const bf16x8* vf = reinterpret_cast<const bf16x8*>(reinterpret_cast<const char*>(vc) + layer * v_layer) + (size_t)chunk * 1024;
  __shared__ bf16 rows[CHUNK * VROW];
  for (int i = t; i < 1024; i += 256) {
    const bf16x8 v = vf[i];
    for (int j = 0; j < 8; j++) rows[vfrag_key(i, j) * VROW + vfrag_d(i)] = v[j];
  }
  __syncthreads();
  for (int i = t; i < 1024; i += 256) {
    const int key = i >> 5, d8 = i & 31, pos = chunk * CHUNK + key;
    if (pos >= tokens) continue;
    bf16x8* k = reinterpret_cast<bf16x8*>(page_row(p, p.d_k, layer, seq, pos));
    bf16x8* v = reinterpret_cast<bf16x8*>(page_row(p, p.d_v, layer, seq, pos));
    if (k == nullptr) continue;
    k[d8] = kf[d8 * 32 + key];
    v[d8] = *reinterpret_cast<const bf16x8*>(&rows[key * VROW + d8 * 8]);
  }
  if (chunk == 0 && layer == 0 && t == 0) p.d_length[seq] = tokens;
}

__global__ __launch_bounds__(256) void pages_load_kernel(pi0_pages p, int seq, bf16* kc, bf16* vc, size_t k_layer, size_t v_layer, int tokens) {
  const int t = threadIdx.x, chunk = blockIdx.x, layer = blockIdx.y;
  bf16x8* kf = reinterpret_cast<bf16x8*>(reinterpret_cast<char*>(kc) + layer * k_layer) + (size_t)chunk * 1024;
  bf16x8* vf = reinterpret_cast<bf16x8*>(reinterpret_cast<char*>(vc) + layer * v_layer) + (size_t)chunk * 1024;
  __shared__ bf16 rows[CHUNK * VROW];
  for (int i = t; i < 1024; i += 256) {
    const int key = i >> 5, d8 = i & 31, pos = chunk * CHUNK + key;
    bf16x8 k = {}, v = {};
    if (pos < tokens) {   // the rest of a chunk is zero: the attention multiplies it by weights of zero
      const bf16x8* kr = reinterpret_cast<const bf16x8*>(page_row(p, p.d_k, layer, seq, pos));
      const bf16x8* vr = reinterpret_cast<const bf16x8*>(page_row(p, p.d_v, layer, seq, pos));
      if (kr != nullptr) k = kr[d8], v = vr[d8];
    }
    kf[d8 * 32 + key] = k;
    *reinterpret_cast<bf16x8*>(&rows[key * VROW + d8 * 8]) = v;
  }
  __syncthreads();
  for (int i = t; i < 1024; i += 256) {
    bf16x8 v;
    for (int j = 0; j < 8; j++) v[j] = rows[vfrag_key(i, j) * VROW + vfrag_d(i)];
    vf[i] = v;
  }
}

bool workspace_ok(const pi0_pages* p, void* ws, size_t bytes, int* rc) {
  if (ws == nullptr || ((uintptr_t)ws & 15) != 0) {
    *rc = PI0_EINVAL;
    return false;
  }
  *rc = PI0_ENOMEM;
  return bytes >= plan_bytes(*p);
}

hipError_t launch_move(hipStream_t s, const pi0_pages& p, const PlanSpace& ws, const int* keep, int keep_stride) {
  const int groups = div_up(p.kv_heads * p.head_dim / 8, MOVE_PIECES);
  return enqueue(s, dim3(groups * p.layers * 2, p.n_seqs), 256, pages_move_kernel, p, ws, keep, keep_stride);
}

}  // namespace

hipError_t launch_pages_store(hipStream_t s, const pi0_pages& p, int seq, const bf16* kc, const bf16* vc, size_t k_layer, size_t v_layer, int tokens) {
  return enqueue(s, dim3(div_up(tokens, CHUNK), p.layers), 256, pages_store_kernel, p, seq, kc, vc, k_layer, v_layer, tokens);
}
hipError_t launch_pages_load(hipStream_t s, const pi0_pages& p, int seq, bf16* kc, bf16* vc, size_t k_layer, size_t v_layer, int tokens) {
  return enqueue(s, dim3(div_up(tokens, CHUNK), p.layers), 256, pages_load_kernel, p, seq, kc, vc, k_layer, v_layer, tokens);
}

extern "C" {

size_t pi0_pages_workspace_bytes(const pi0_pages* pages) { return pages_ok(pages) ? plan_bytes(*pages) : 0; }

int pi0_pages_reserve(const pi0_pages* pages, const int32_t* d_extra, void* d_workspace, size_t ws_bytes, void* hip_stream) {
  int rc = PI0_EINVAL;
  if (!pages_ok(pages) || d_extra == nullptr || !workspace_ok(pages, d_workspace, ws_bytes, &rc)) return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  PlanArgs a = {};
  a.p = *pages;
  a.ws = plan_space(*pages, d_workspace);
  a.extra = d_extra;
  hipError_t e = enqueue(s, dim3(1), PLAN_THREADS, pages_plan_kernel<PLAN_RESERVE>, a);
  if (e == hipSuccess) e = launch_move(s, *pages, a.ws, nullptr, 0);
  return e == hipSuccess ? PI0_OK : PI0_EHIP;
}

int pi0_pages_compact(const pi0_pages* pages, const int32_t* d_start, const int32_t* d_keep, int keep_stride, const int32_t* d_n_keep,
                      void* d_workspace, size_t ws_bytes, void* hip_stream) {
  int rc = PI0_EINVAL;
  if (!pages_ok(pages) || d_n_keep == nullptr || keep_stride < 0 || (keep_stride > 0 && d_keep == nullptr) ||
      !workspace_ok(pages, d_workspace, ws_bytes, &rc))
    return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  PlanArgs a = {};
  a.p = *pages;
  a.ws = plan_space(*pages, d_workspace);
  a.start = d_start;
  a.keep = d_keep;
  a.n_keep = d_n_keep;
  a.keep_stride = keep_stride;
  hipError_t e = enqueue(s, dim3(1), PLAN_THREADS, pages_plan_kernel<PLAN_COMPACT>, a);
  if (e == hipSuccess) e = launch_move(s, *pages, a.ws, d_keep, keep_stride);
  return e == hipSuccess ? PI0_OK : PI0_EHIP;
}

int pi0_pages_fork(const pi0_pages* pages, const int32_t* d_src, const int32_t* d_dst, int n, void* hip_stream) {
  if (!pages_ok(pages) || d_src == nullptr || d_dst == nullptr || n < 1 || n > pages->n_seqs) return PI0_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  return enqueue(s, dim3(1), PLAN_THREADS, pages_fork_kernel, *pages, d_src, d_dst, n) == hipSuccess ? PI0_OK : PI0_EHIP;
}

int pi0_pages_status(const pi0_pages* pages, void* hip_stream) {
  if (!pages_ok(pages)) return PI0_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  int32_t code = 0, none = 0;
  hipError_t e = hipMemcpyAsync(&code, pages->d_status, sizeof code, hipMemcpyDeviceToHost, s);
  if (e == hipSuccess) e = hipStreamSynchronize(s);
  if (e == hipSuccess && code != 0) {
    e = hipMemcpyAsync(pages->d_status, &none, sizeof none, hipMemcpyHostToDevice, s);
    if (e == hipSuccess) e = hipStreamSynchronize(s);
  }
  return e == hipSuccess ? code : PI0_EHIP;
}

}  // extern "C"
