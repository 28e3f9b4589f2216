// Paged K/V cache: arguments of the kernels, and the index arithmetic they share with the host (compiles without CUDA).
#pragma once
#include <stdint.h>

#if defined(__CUDACC__)
#define FC_ANY __host__ __device__ __forceinline__
#else
#define FC_ANY inline
#endif

namespace fc {

// One layer of a pool, strides in elements.
struct PageView {
  void *k, *v;
  long long page_stride, head_stride, slot_stride;
  int n_pages, page_size, n_kv_heads;
};

struct PagedAttnArgs {
  PageView pool;
  const int32_t *table; int width;
  int cap;                // positions of a table row: width x page_size
  const int32_t *kv_len;
  const void *q; long long q_stride;      // elements
  float *out;             // [batch * c, hq * hd]
  int batch, c, hq, window, n_sink;       // n_sink is 0 without a window
  // set by the launcher: the queries' arithmetic (reciprocal of the heads of a group), the pool's strides in bytes
  int group, nq, groups;  // heads of a group, queries of a kv head, units of a kv head
  unsigned int group_inv;
  int hd, elem_bytes;
  long long page_bytes, head_bytes, slot_bytes;
  float *parts;           // scratch: two parts per worker, [queries][hd] sums and [queries] (max, sum)
  unsigned int *status;   // scratch of the kernel that has waits, else null: per worker, 1 where a wait ran out
};

// Length of a sequence as the kernels use it: -1 for none, never far beyond the table's `cap` positions (no sum overflows).
FC_ANY int clamp_len(int len, int cap) { return len < 0 ? -1 : len > cap ? cap : len; }

// Page of position t, -1 if there is none in the pool.  row: the sequence's entries of the table.
FC_ANY int page_of(const int32_t *row, int width, int t, int page_size, int n_pages) {
  if (t < 0) return -1;
  const int i = t / page_size;
  if (i >= width) return -1;
  const int p = row[i];
  return p >= 0 && p < n_pages ? p : -1;
}

// Whether the row at position p sees the key at position t >= 0.
FC_ANY bool sees(int p, int t, int window, int n_sink) { return t <= p && (window == 0 || t > p - window || t < n_sink); }

// First position that a row at position p sees because of the window.
FC_ANY int window_first(int p, int window) { return window == 0 || p < window ? 0 : p - window + 1; }

// Whether entry i of a table is released under a sliding window: no row at position len or later sees a slot of it.
FC_ANY bool page_unseen(int i, int page_size, int len, int window, int n_sink) {
  return (long long)(i + 1) * page_size <= (long long)len - window + 1 && (long long)i * page_size >= n_sink;
}

// The keys that some of the rows at positions len .. len + rows - 1 see, in tiles of `keys` positions: tiles 0 .. sinks - 1, then
// first .. first + n - sinks - 1.  Rows beyond the table see what is in it (their result is NaN whatever that is).
struct KeyTiles { int n, sinks, first; };
FC_ANY KeyTiles key_tiles(int len, int rows, int cap, int window, int n_sink, int keys) {
  KeyTiles t = {0, 0, 0};
  if (len < 0) return t;
  const int last = (len + rows < cap ? len + rows : cap) - 1;
  int low = window_first(len, window);
  if (low > last) low = last;
  const unsigned int k = (unsigned int)keys;             // a power of two that the compiler knows, where it matters
  t.first = (int)((unsigned int)low / k);
  const int sink_keys = window == 0 ? 0 : n_sink < low ? n_sink : low;
  t.sinks = (int)(((unsigned int)sink_keys + k - 1) / k);
  if (t.sinks > t.first) t.sinks = t.first;
  t.n = t.sinks + (int)((unsigned int)last / k) - t.first + 1;
  return t;
}
FC_ANY int tile_key(const KeyTiles &t, int i, int keys) { return (i < t.sinks ? i : t.first + i - t.sinks) * keys; }

// All tiles of a launch stand in one line (its host side sees to it that they are fewer than 2^31): sequence by sequence, unit (kv head,
// group of queries) by unit, and each of `workers` takes `chunk` of them in a row.  The parts of the unit at [begin, begin + n) and where worker i left its part: place 0 for what a
// worker begins with, 1 for what it ends with.
// A part: [queries][hd] sums, then [queries] (max, sum), in whole 16-byte pieces (sums are written and read four at a time).
FC_ANY constexpr int part_floats(int queries, int hd) { return queries * hd + (2 * queries + 3) / 4 * 4; }
struct UnitParts { int first, last; };
FC_ANY int chunk_of(int total, int workers) { return total / workers + (total % workers != 0); }
FC_ANY UnitParts unit_parts(int begin, int n, int chunk) {
  const int first = (int)((unsigned int)begin / (unsigned int)chunk);
  return {first, first + (int)((unsigned int)(begin - first * chunk + n - 1) / (unsigned int)chunk)};
}
FC_ANY int part_place(int begin, int worker, int chunk) { return begin > worker * chunk; }

// x / n for 0 <= x < 2^16, n < 2^16, by the reciprocal of n.
FC_ANY unsigned int reciprocal16(int n) { return n == 1 ? 0u : (unsigned int)((0x100000000ull + (unsigned int)n - 1) / (unsigned int)n); }
FC_ANY int quotient16(int x, unsigned int inv) { return inv ? (int)((unsigned long long)(unsigned int)x * inv >> 32) : x; }

// Sequences that a launch can take: units of each in at most the table's tiles; 0 if not even one.
inline int line_batch(int units, int cap, int keys) {
  const long long most = (long long)units * (cap / keys + 1);
  return most > 0x7fffffff ? 0 : (int)(0x7fffffffll / most);
}

// CTAs of a cluster per unit where one launch of clusters does the work of the line and the kernel that joins its parts, 0 otherwise.  All
// clusters have to run at once, and no warp may have more than a few tiles, whatever the lengths are (only the table's bound on them is known).
inline int paged_cluster(int batch, int units, int cap, int c, int window, int n_sink, int keys, int warps, int sms) {
  const long long most = window > 0 && (long long)window + c + n_sink < cap ? (long long)window + c + n_sink + 2 * keys : cap;
  const long long tiles = (most + keys - 1) / keys;
  int ctas = 1;
  while (ctas < 8 && tiles > ctas * warps && (long long)batch * units * ctas * 2 <= sms - 20) ctas *= 2;
  return (long long)batch * units * ctas <= sms && tiles <= 4ll * warps * ctas ? ctas : 0;
}

// Whether the kernel on tcgen05 takes a kv head's nq queries.
inline bool paged_umma(int nq, int hd) { return nq > 32 && hd >= 64; }
// Queries of a unit and keys of a tile in fp32 (k_paged_fma.cu) and in bf16 (k_paged_attn.cu, k_paged_umma.cu).
inline int paged_queries(int nq, int hd, bool f32) { return f32 ? (nq == 1 ? 1 : 8) : paged_umma(nq, hd) ? 128 : nq <= 8 ? 8 : 16; }
inline int paged_keys(int nq, int hd, bool f32) { return f32 ? 1024 / hd : paged_umma(nq, hd) ? 64 : 16; }
// Whether one sequence's tiles can be counted.
inline bool paged_line_fits(int nq, int n_kv_heads, int hd, bool f32, int cap) {
  const int q = paged_queries(nq, hd, f32);
  return line_batch(n_kv_heads * ((nq + q - 1) / q), cap, paged_keys(nq, hd, f32)) > 0;
}

}  // namespace fc
