// The paged cache as kernels see it, shared by the pages' own operations and by the attention that reads them.
#pragma once
#include "asl_internal.cuh"

// asl_pages_*, checked: ASL_OK, or why the description cannot be used.
asl_status asl_check_pages(const asl_pages* p);
// Kernels go to the thread's current device, which has to be the context's.
inline bool asl_on_device(const asl_ctx* c) {
  int device = -1;
  return cudaGetDevice(&device) == cudaSuccess && device == c->device;
}
inline bool asl_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct PagePool {
  uint8_t* k;              // of one layer
  uint8_t* v;
  int32_t* table;
  int32_t* len;
  int32_t* refs;
  int32_t* err;
  int32_t n_pages, max_seqs, max_pages, page_shift, n_kv_heads;
  int32_t k_row, v_row;    // bytes of a row
};

inline int page_shift_of(int page_size) { return page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : 7; }

inline PagePool page_pool(const asl_pages* p, int layer) {
  PagePool g;
  g.k_row = p->head_dim * (p->k_dtype == ASL_K_FP8_E4M3 ? 1 : 2);
  g.v_row = p->head_dim * 2;
  const int64_t rows = (int64_t)p->n_pages * p->n_kv_heads * p->page_size;
  g.k = static_cast<uint8_t*>(p->k) + rows * g.k_row * layer;
  g.v = static_cast<uint8_t*>(p->v) + rows * g.v_row * layer;
  g.table = p->table;
  g.len = p->len;
  g.refs = p->refs;
  g.err = p->err;
  g.n_pages = p->n_pages;
  g.max_seqs = p->max_seqs;
  g.max_pages = p->max_pages;
  g.page_shift = page_shift_of(p->page_size);
  g.n_kv_heads = p->n_kv_heads;
  return g;
}

#ifdef __CUDACC__
__device__ __forceinline__ void note_error(int32_t* err, int code, int info) {
  if (atomicCAS(err, 0, code) == 0) err[1] = info;
}
__device__ __forceinline__ int pages_for(int tokens, int shift) { return (tokens + (1 << shift) - 1) >> shift; }
#endif
