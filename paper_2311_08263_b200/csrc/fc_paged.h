// Paged K/V cache: arguments of the kernels, and the index arithmetic they share with the host (compiles without CUDA).
#pragma once
#include <stdint.h>

#if defined(__CUDACC__)
#define FC_HD __host__ __device__ __forceinline__
#else
#define FC_HD inline
#endif

namespace fc {

// One layer of a pool, strides in elements.
struct PageView {
  void *k, *v;
  long long page_stride, head_stride, slot_stride;
  int n_pages, page_size, n_kv_heads;
};

// Length of a sequence as the kernels use it: -1 for none, never far beyond the table's `cap` positions (no sum overflows).
FC_HD int clamp_len(int len, int cap) { return len < 0 ? -1 : len > cap ? cap : len; }

// Page of position t, -1 if there is none in the pool.  row: the sequence's entries of the table.
FC_HD int page_of(const int32_t *row, int width, int t, int page_size, int n_pages) {
  if (t < 0) return -1;
  const int i = t / page_size;
  if (i >= width) return -1;
  const int p = row[i];
  return p >= 0 && p < n_pages ? p : -1;
}

// Whether the row at position p sees the key at position t >= 0.
FC_HD bool sees(int p, int t, int window, int n_sink) { return t <= p && (window == 0 || t > p - window || t < n_sink); }

// First position that a row at position p sees because of the window.
FC_HD int window_first(int p, int window) { return window == 0 || p < window ? 0 : p - window + 1; }

// Whether entry i of a table is released under a sliding window: no row at position len or later sees a slot of it.
FC_HD bool page_unseen(int i, int page_size, int len, int window, int n_sink) {
  return (long long)(i + 1) * page_size <= (long long)len - window + 1 && (long long)i * page_size >= n_sink;
}

}  // namespace fc
