// Paged K/V cache: arguments of the kernels, and the index arithmetic they share with the host (compiles without CUDA).
#pragma once
#include <stddef.h>
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
  int hd, elem_bytes, first;      // first: the sequence of the call that this launch begins with
  long long page_bytes, head_bytes, slot_bytes;
  float *parts;           // scratch: two parts per worker, [queries][hd] sums and [queries] (max, sum)
  unsigned int *status;   // scratch of the kernel that has waits, else null: per worker, 1 where a wait ran out
};

// Elements of a page are counted in 32 bits.
FC_ANY bool page_too_large(int n_kv_heads, int page_size, int hd) { return (long long)n_kv_heads * page_size > (1ll << 31) / hd; }

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

// Where a line's tiles are loaded by copies, kCopyWarps warps take turns at them (k_paged_umma.cu).  The queries of a segment go into one of two places,
// behind the products of the segment but one in front of it, for which the loading warp waits with a parity: that tells a phase only from the ones next to it,
// so the warp must have waited for all phases before.  Hence one warp loads the queries of all segments, whoever copies their first tile.
constexpr int kCopyWarps = 2;
FC_ANY int query_copier(int first_tile) { return 0; }

// x / n for 0 <= x < 2^16, n < 2^16, by the reciprocal of n.
FC_ANY unsigned int reciprocal16(int n) { return n == 1 ? 0u : (unsigned int)((0x100000000ull + (unsigned int)n - 1) / (unsigned int)n); }
FC_ANY int quotient16(int x, unsigned int inv) { return inv ? (int)((unsigned long long)(unsigned int)x * inv >> 32) : x; }

// Sequences that a launch can take: units of each in at most the table's tiles; 0 if not even one.
inline int line_batch(int units, int cap, int keys) {
  const long long most = (long long)units * (cap / keys + 1);
  return most > 0x7fffffff ? 0 : (int)(0x7fffffffll / most);
}

// ---- which kernel a call takes, and in which form
// kFma: fp32 (k_paged_fma.cu); kMma: bf16 (k_paged_attn.cu); kUmma: bf16 on tcgen05 (k_paged_umma.cu).
enum PagedKind { kFma, kMma, kUmma };
struct PagedPlan {
  PagedKind kind;
  int queries, keys;      // of a unit, of a tile
  int units;              // of a sequence
  int ctas;               // CTAs of a cluster per unit; 0: the line
  int workers;            // of the line
  size_t scratch;         // bytes; 0 with clusters
  bool fits;              // one sequence's tiles can be counted
};
constexpr int kPagedSms = 148, kPagedWarps = 8, kMoreWarps = 12, kUmmaQueries = 128, kUmmaKeys = 64, kMmaKeys = 16;
constexpr size_t kUmmaStatus = (kPagedSms * sizeof(unsigned int) + 255) / 256 * 256;

// CTAs of a cluster per unit where one launch of clusters does the work of the line and the kernel that joins its parts, 0 otherwise.  All
// clusters have to run at once, and no warp may have more than a few tiles, whatever the lengths are (only the table's bound on them is known).
inline int paged_cluster(int batch, int units, long long most_keys, int keys) {
  const long long tiles = (most_keys + keys - 1) / keys;
  int ctas = 1;
  while (ctas < 8 && tiles > ctas * kPagedWarps && (long long)batch * units * ctas * 2 <= kPagedSms - 20) ctas *= 2;
  return (long long)batch * units * ctas <= kPagedSms && tiles <= 4ll * kPagedWarps * ctas ? ctas : 0;
}

// Whether tcgen05 pays: its units are 128 queries, used or not, and it starts and ends slowly.  By what both cost (microseconds, keys up to the
// table's bound): 5 and 0.168 (hd 64) or 0.232 (hd 128) per 16 queries x 16 keys and SM, against 12 and 1.09 or 2.3 per unit's tile of 64 keys and SM.
// Measured, mma.sync against tcgen05, sequences x kv heads x queries: hd 128, 4 x 32 x 64 over 1000 keys 61.7, 43.7; 8 x 8 x 64 over 2000 58.5, 41.9; 8 x 40 x 64 over
// 1024 135, 95.5; 1 x 8 x 128 over 4000 37.0, 31.8; 1 x 8 x 64 over 4000 25.0, 28.4; 1 x 8 x 128 over 1000 13.3, 19.7; hd 64, 16 x 4 x 128 over 4000 105, 36.8,
// over 641 27.7, 20.8; 8 x 4 x 64 over 2000 23.6, 21.1; 4 x 4 x 128 over 641 15.1, 16.4; 1 x 4 x 128 over 641 7.7, 12.7.  (Chosen wrongly by up to 10 %: hd 128, 2 x 8 x 64
// over 2000 23.6, 22.0; 4 x 8 x 128 over 500 27.5, 30.3.)  All of that in tables as wide as their caches: only the table's width is known here, and a table for much
// more than its sequences hold gets the form for long ones (hd 64, 1 x 4 x 128 over 641 keys in a table for 4096
// positions: 12.7 us on tcgen05, 7.5 in clusters in one for 2048).
inline bool umma_pays(int batch, int n_kv_heads, int nq, int hd, long long most_keys) {
  if (nq <= 32 || hd < 64) return false;
  const double heads = (double)batch * n_kv_heads / kPagedSms;
  const double mma = 5 + heads * ((nq + 15) / 16) * (most_keys / 16.0) * (hd == 128 ? 0.232 : 0.168);
  const double umma = 12 + heads * ((nq + 127) / 128) * (most_keys / 64.0) * (hd == 128 ? 2.3 : 1.09);
  return umma < mma;
}

// Warps per SM on the line of k_paged_attn.cu: more of them hide each other's waits where there is much to do; where there is little they leave more parts.  Measured,
// 8 and 12 warps, by tiles per warp of 8: 7 (1 sequence x 4 kv heads over 32000 keys, hd 64) 14.5, 16.5 us; 5.5 (4 x 32 x 16 queries over 800, hd 128) 22.5, 24.1; 13.5 (8 x 8 over
// 4000) 30.2, 29.7; 18 (8 x 40 x 16 over 1024) 50.9, 48.4; 35 (8 x 40 x 4 over 2052) 61.8, 59.8.  (10 warps 53.8 and 60.7; 16, at hd 64, as 12 or slower.)
inline bool more_warps_pay(long long units, long long most_keys) { return units * (most_keys / kMmaKeys) >= 10ll * kPagedSms * kPagedWarps; }

inline PagedPlan paged_plan(int batch, int c, int hq, int hkv, int hd, bool f32, int cap, int window, int n_sink) {
  PagedPlan p;
  const int nq = hq / hkv * c;
  const long long bound = (long long)window + c + n_sink + 2 * kMmaKeys, most = window > 0 && bound < cap ? bound : cap;      // keys of a sequence
  p.kind = f32 ? kFma : umma_pays(batch, hkv, nq, hd, most) ? kUmma : kMma;
  p.queries = p.kind == kUmma ? kUmmaQueries : p.kind == kFma && nq == 1 ? 1 : p.kind == kFma || nq <= 8 ? 8 : 16;
  p.keys = p.kind == kUmma ? kUmmaKeys : p.kind == kFma ? 1024 / hd : kMmaKeys;
  p.units = hkv * ((nq + p.queries - 1) / p.queries);
  p.ctas = p.kind == kUmma ? 0 : paged_cluster(batch, p.units, most, p.keys);
  p.workers = kPagedSms * (p.kind == kUmma ? 1 : p.kind == kMma && more_warps_pay((long long)batch * p.units, most) ? kMoreWarps : kPagedWarps);
  p.scratch = p.ctas ? 0 : (p.kind == kUmma ? kUmmaStatus : 0) + (size_t)p.workers * 2 * part_floats(p.queries, hd) * sizeof(float);
  p.fits = line_batch(p.units, cap, p.keys) > 0;
  return p;
}

}  // namespace fc
