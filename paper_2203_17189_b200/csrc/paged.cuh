// Shared declarations of the paged key / value cache: where a key lives, the status codes, argument checks.
#pragma once
#include "common.cuh"

#include <string.h>

// Status codes the kernels of the paged cache leave in the word of t5_kernel_status_word (first one wins)
enum { PAGED_BAD_APPEND = 201, PAGED_BAD_PAGE = 202, PAGED_BAD_LENGTH = 203, PAGED_TIMEOUT = 204 };

__device__ __forceinline__ void paged_report(int* status, int code) {
  if (status != nullptr) atomicCAS(status, 0, code);
}

// n / d for 0 <= n < 2^31 by one multiplication: with s = ceil(log2 d), m = ceil(2^(31+s) / d) < 2^32 and
// n m / 2^(31+s) exceeds n / d by less than n / 2^31 / d * (m d - 2^(31+s)) / 2^s < 1 / d, so the floor is exact.
struct FastDiv {
  uint32_t d, m, s;
  FastDiv() = default;
  __host__ explicit FastDiv(uint32_t dd) : d(dd), m(0), s(0) {      // 0: never divided by
    while ((1ull << s) < d) ++s;
    if (s > 0) m = (uint32_t)(((1ull << (31 + s)) + d - 1) / d);
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return s == 0 ? n : __umulhi(n, m) >> (s - 1); }
};

// Page pools: element (page, slot, head, c) of K at k + (page * page_stride + slot * slot_stride + head * head_stride + c)
// elements, V alike; sequence s finds its key j in page table[s * ld_table + j / page_size], slot j % page_size.
// Strides are held in bytes here.
struct PagedPool {
  char *k, *v;
  int n_pages, page_size;
  int64_t page_stride, slot_stride, head_stride;
  const int* table;
  int64_t ld_table;
  int max_pages;
  FastDiv ps;
};

// Code of a launch; the runtime's record of a failed one is cleared, so that the next call does not report it again
inline int paged_result(cudaError_t e) {
  if (e == cudaSuccess) return 0;
  cudaGetLastError();
  return -6;      // T5_ERR_CUDA
}
inline bool paged_aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Checks shared by the calls that take pools; fills `out`.  Returns a T5_ERR_* code.
int paged_pool_args(int es, int n_kv_heads, int d_kv, const void* k_pages, const void* v_pages, int n_pages, int page_size,
                    int64_t page_stride, int64_t slot_stride, int64_t head_stride, const int* table, int n_seqs,
                    int max_pages, int64_t ld_table, PagedPool* out);

// Launchers used by the entry points and by the model's paged decoding step
struct PagedAppendArgs {
  int dtype, n_tokens, n_heads, n_kv_heads, d_kv;
  const void *q, *k, *v;
  void* q_out;
  int64_t ldq, ldk, ldv, ldqo;      // elements
  const int *seq, *pos;             // seq NULL: token t belongs to sequence t / tokens_per_seq
  int tokens_per_seq;
  int rot_dim, interleaved;
  double rot_base;
  PagedPool pool;
  int n_seqs;
  int* status;
};
cudaError_t launch_paged_append(const PagedAppendArgs& a, cudaStream_t st);

struct PagedAttnArgs {
  int dtype, n_rows, n_q, H, Hkv, d_kv;
  const void* q;
  void* out;
  int64_t ldq, ldo;                 // elements
  float* lse;                       // [n_rows, H] or NULL
  const int* lens;                  // [n_rows]
  const float* bias;                // [H, n_bias] or NULL: entry n_bias - 1 - distance, saturating at entry 0
  int n_bias;
  float scale;
  PagedPool pool;
  void* workspace;
  int* status;
};
int64_t paged_attention_workspace(int n_rows, int n_q, int H, int Hkv, int d_kv);
cudaError_t launch_paged_attention(const PagedAttnArgs& a, cudaStream_t st);
bool paged_attention_tc_fits(const PagedAttnArgs& a);      // many query rows per kv head, of a form that kernel takes
cudaError_t launch_paged_attention_tc(const PagedAttnArgs& a, cudaStream_t st);
