// Declarations shared by the operators on a paged key/value cache (pages.hip, qk_norm_rope.hip, tree_attention.hip).
#pragma once
#include "pi0_internal.h"
#include "../../include/pi0_ops.h"

typedef _Float16 f16;

constexpr int MAX_SEQS = 1024;   // sequences of a cache

// what the host can check of a cache without looking at device memory
bool pages_ok(const pi0_pages* p);
// rows of `heads` heads (0: any number) of `head_dim` elements in type `dtype`
bool rows_ok(const pi0_rows* r, int heads, int head_dim, int dtype);

// A launch and its own result: hipGetLastError would give back an error that an earlier call of the caller's left, too.
template <class T>
struct Same { typedef T type; };
template <class... P>
static inline hipError_t enqueue(hipStream_t s, dim3 grid, int threads, void (*kernel)(P...), const typename Same<P>::type&... arg) {
  void* args[] = {const_cast<void*>(static_cast<const void*>(&arg))...};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), args, 0, s);
  if (e != hipSuccess) (void)hipGetLastError();   // told by what is returned
  return e;
}

static __host__ __device__ __forceinline__ int div_up(int a, int b) { return (a + b - 1) / b; }

// the page behind entry `idx` of a sequence's list, or -1
static __device__ __forceinline__ int page_at(const pi0_pages& p, int seq, int idx) {
  if (idx < 0 || idx >= p.max_pages) return -1;
  const int page = p.d_table[(size_t)seq * p.max_pages + idx];
  return page >= 0 && page < p.n_pages ? page : -1;
}

// A sequence's new tokens: first row and number, from what the caller's row_start says, inside [0, n_rows) and at most max_rows.
static __device__ __forceinline__ int2 rows_of(const int* row_start, int seq, int n_rows, int max_rows) {
  const int first = row_start[seq], end = min(row_start[seq + 1], n_rows);
  if (first < 0 || first >= end) return make_int2(0, 0);
  return make_int2(first, min(end - first, max_rows));
}

// committed positions of a sequence, never more than its table can name
static __device__ __forceinline__ int length_of(const pi0_pages& p, int seq) {
  return max(0, min(p.d_length[seq], p.max_pages * p.page_tokens));
}

// pi0_api.hip's part of pi0_pages_store / pi0_pages_load: one layer's keys and values lie `k_layer`, `v_layer` bytes behind the other's
hipError_t launch_pages_store(hipStream_t s, const pi0_pages& p, int seq, const bf16* kc, const bf16* vc, size_t k_layer, size_t v_layer, int tokens);
hipError_t launch_pages_load(hipStream_t s, const pi0_pages& p, int seq, bf16* kc, bf16* vc, size_t k_layer, size_t v_layer, int tokens);
