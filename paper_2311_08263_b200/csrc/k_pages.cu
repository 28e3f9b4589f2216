// Pages of a K/V pool: sharing, copy on write, release, compaction.
//
// Tables, lengths and reference counts live on the device and every decision is made there, so that a serving loop can be captured.  What
// is decided per call is small (a few entries per sequence, one pass over the counts): one block, whose scans make every choice
// deterministic: the k-th page that is needed, by table row, is the k-th lowest free one.  What costs is copying pages, in all layers:
// 2 x bytes of the pages moved, bound by HBM.
#include <climits>
#include <cstring>
#include <new>

#include "fc_internal.h"
#include "fc_paged.h"

namespace fc {

namespace {

constexpr int kPlanThreads = 1024;
// Table rows named in one launch's parameters: a few, or many (large parameters cost the launch about a microsecond).
constexpr int kListed = 500, kFew = 32;
template <int N> struct SeqList { int a[N], b[N]; };

// ------------------------------------------------------------------------------------------------ free, fork
__device__ __forceinline__ void release(int32_t *refs, int n_pages, int e) {
  if (e >= 0 && e < n_pages) atomicSub(refs + e, 1);
}

template <int N>
__global__ void __launch_bounds__(128) pages_free_kernel(int32_t *table, int width, int32_t *kv_len, int32_t *refs, int n_pages, int page_size,
                                                        const __grid_constant__ SeqList<N> list, int window, int n_sink) {
  const int s = list.a[blockIdx.x];
  int32_t *row = table + (long long)s * width;
  const int len = kv_len[s];
  for (int i = threadIdx.x; i < width; i += 128) {
    if (window > 0 && !page_unseen(i, page_size, len, window, n_sink)) continue;
    release(refs, n_pages, row[i]);
    row[i] = -1;
  }
  __syncthreads();
  if (window == 0 && threadIdx.x == 0) kv_len[s] = -1;
}

template <int N>
__global__ void __launch_bounds__(128) pages_fork_kernel(int32_t *table, int width, int32_t *kv_len, int32_t *refs, int n_pages, int page_size,
                                                        const __grid_constant__ SeqList<N> list) {
  const int src = list.a[blockIdx.x], dst = list.b[blockIdx.x];
  const int32_t *from = table + (long long)src * width;
  int32_t *to = table + (long long)dst * width;
  const int len = kv_len[src];
  const int held = len <= 0 ? 0 : (len - 1) / page_size + 1;           // pages with committed tokens
  for (int i = threadIdx.x; i < width; i += 128) {
    int e = i < held ? from[i] : -1;
    if (e < 0 || e >= n_pages) e = -1;
    else atomicAdd(refs + e, 1);
    release(refs, n_pages, to[i]);
    to[i] = e;
  }
  if (threadIdx.x == 0) kv_len[dst] = len < 0 ? -1 : len;
}

// ------------------------------------------------------------------------------------------------ scans of one block
// Exclusive sum over the block's threads; *all: the sum.
__device__ __forceinline__ int block_scan(int v, int *all) {
  __shared__ int part[kPlanThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) part[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int w = part[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += y;
    }
    part[lane] = w;
  }
  __syncthreads();
  *all = part[kPlanThreads / 32 - 1];
  return x - v + (warp ? part[warp - 1] : 0);
}

// ------------------------------------------------------------------------------------------------ reserve
struct ReserveArgs {
  int32_t *table; int width, n_seqs;
  const int32_t *kv_len;
  int32_t *refs; int n_pages, page_size, rows;
  int32_t *served;
  // scratch: per page writers, keeper, free pages in order; per sequence its copy; how many copies
  int32_t *writers, *keeper, *free_list, *src, *dst, *n_copies;
};

// Table entries that sequence b writes: [first, first + n); n = 0 where there is no sequence, -1 where the table is too short.
__device__ __forceinline__ int write_range(const ReserveArgs &a, int b, int &first, int &len) {
  len = a.kv_len[b];
  first = 0;
  if (len < 0) return 0;
  const long long end = ((long long)len + a.rows - 1) / a.page_size;
  if (end >= a.width) return -1;
  first = len / a.page_size;
  return (int)end - first + 1;
}
__device__ __forceinline__ int held_page(const ReserveArgs &a, int b, int i) {
  const int e = a.table[(long long)b * a.width + i];
  return e >= 0 && e < a.n_pages ? e : -1;
}

__global__ void __launch_bounds__(kPlanThreads) pages_reserve_kernel(const __grid_constant__ ReserveArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");       // the copies wait until this is done
  const int tid = threadIdx.x;
  __shared__ int copies;
  if (tid == 0) copies = 0;
  // who writes the pages that are there: how many sequences, and the last of them
  for (int step = 0; step < 3; ++step) {
    for (int b = tid; b < a.n_seqs; b += kPlanThreads) {
      int first, len;
      const int n = write_range(a, b, first, len);
      for (int i = 0; i < n; ++i) {
        const int p = held_page(a, b, first + i);
        if (p < 0) continue;
        if (step == 0) { a.writers[p] = 0; a.keeper[p] = -1; }
        else if (step == 1) { atomicAdd(a.writers + p, 1); atomicMax(a.keeper + p, b); }
        else if (a.writers[p] != a.refs[p]) a.keeper[p] = -1;           // somebody else holds it: nobody keeps it
      }
    }
    __syncthreads();
  }
  // what each sequence needs, and where its pages begin in the list of free ones
  int want = 0;
  for (int b0 = 0; b0 < a.n_seqs; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int need = 0, first, len, all;
    if (b < a.n_seqs) {
      const int n = write_range(a, b, first, len);
      for (int i = 0; i < n; ++i) {
        const int p = held_page(a, b, first + i);
        need += p < 0 || a.keeper[p] != b;
      }
    }
    const int before = block_scan(need, &all);
    if (b < a.n_seqs) { a.src[b] = want + before; a.dst[b] = need; }
    want += all;
  }
  // the lowest free pages, as many as are wanted
  int found = 0;
  for (int p0 = 0; p0 < a.n_pages && found < want; p0 += kPlanThreads) {
    const int p = p0 + tid;
    const int is_free = p < a.n_pages && a.refs[p] <= 0;
    int all;
    const int at = found + block_scan(is_free, &all);
    if (is_free && at < want) a.free_list[at] = p;
    found += all;
  }
  __syncthreads();
  // sequences in order, as far as the pages last (the first that does not get its pages ends it for all behind it)
  for (int b = tid; b < a.n_seqs; b += kPlanThreads) {
    int first, len;
    const int n = write_range(a, b, first, len);
    int at = a.src[b];
    const int need = a.dst[b];
    const bool ok = n > 0 && at + need <= found;
    if (a.served) a.served[b] = ok;
    if (!ok) continue;
    for (int i = 0; i < n; ++i) {
      const int p = held_page(a, b, first + i);
      if (p >= 0 && a.keeper[p] == b) continue;
      const int fresh = a.free_list[at++];
      a.refs[fresh] = 1;
      if (p >= 0) {
        atomicSub(a.refs + p, 1);
        if (i == 0 && len % a.page_size) {                              // committed tokens in it
          const int k = atomicAdd(&copies, 1);
          a.free_list[a.n_pages + k] = p;
          a.free_list[a.n_pages + a.n_seqs + k] = fresh;
        }
      }
      a.table[(long long)b * a.width + first + i] = fresh;
    }
  }
  __syncthreads();
  if (tid == 0) *a.n_copies = copies;
}

// ------------------------------------------------------------------------------------------------ compact
struct CompactArgs {
  int32_t *refs; int n_pages;
  int32_t *n_live;                          // of the caller, or null
  int32_t *dst, *src, *place, *counts;      // scratch: holes, pages that move, where each page from n on goes; how many move, how many live
};

__global__ void __launch_bounds__(kPlanThreads) pages_compact_kernel(const __grid_constant__ CompactArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");       // the copies wait until this is done
  const int tid = threadIdx.x;
  int live = 0, all;
  for (int p = tid; p < a.n_pages; p += kPlanThreads) live += a.refs[p] > 0;
  block_scan(live, &all);
  const int n = all;
  int holes = 0, high = 0;
  for (int p0 = 0; p0 < a.n_pages; p0 += kPlanThreads) {
    const int p = p0 + tid;
    const bool used = p < a.n_pages && a.refs[p] > 0;
    const int is_hole = p < n && !used, is_high = p >= n && used;
    int all_h, all_l;
    const int at_h = block_scan(is_hole, &all_h), at_l = block_scan(is_high, &all_l);
    if (is_hole) a.dst[holes + at_h] = p;
    if (is_high) a.src[high + at_l] = p;
    if (p >= n && p < a.n_pages && !used) a.place[p] = -1;
    holes += all_h;
    high += all_l;
  }
  __syncthreads();
  for (int i = tid; i < high; i += kPlanThreads) {
    const int from = a.src[i], to = a.dst[i];
    a.place[from] = to;
    a.refs[to] = a.refs[from];
    a.refs[from] = 0;
  }
  if (tid == 0) {
    a.counts[0] = high;
    a.counts[1] = n;
    if (a.n_live) *a.n_live = n;
  }
}

// ------------------------------------------------------------------------------------------------ copies
struct CopyArgs {
  uint4 *k, *v;
  const int32_t *src, *dst, *n;             // pages, device
  long long layer_stride, page_stride;      // in 16-byte pieces, as all below
  int n_layers;
  unsigned int piece;                       // pieces of a page in one layer's keys (or values)
  // a page as runs of `run` adjacent pieces: run i at (i / inner) * outer_stride + (i % inner) * inner_stride
  unsigned int run, inner;
  long long inner_stride, outer_stride;
  // compaction: the table that follows (null: none)
  int32_t *table; long long entries;
  const int32_t *place, *n_live; int n_pages;
};

constexpr int kCopyThreads = 256, kCopyUnroll = 4;

__global__ void __launch_bounds__(kCopyThreads) pages_copy_kernel(const __grid_constant__ CopyArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");                    // the kernel that decided what is copied
  const int n = *a.n;
  const unsigned int chunk = kCopyThreads * kCopyUnroll, chunks = (a.piece + chunk - 1) / chunk;
  const long long units = (long long)n * a.n_layers * 2 * chunks;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    long long r = u / chunks;
    const unsigned int c0 = (unsigned int)(u - r * chunks) * chunk + threadIdx.x;
    uint4 *base = (r & 1) ? a.v : a.k;
    r >>= 1;
    const int layer = (int)(r % a.n_layers), i = (int)(r / a.n_layers);
    base += layer * a.layer_stride;
    const uint4 *from = base + (long long)a.src[i] * a.page_stride;
    uint4 *to = base + (long long)a.dst[i] * a.page_stride;
    uint4 x[kCopyUnroll];
    long long at[kCopyUnroll];
#pragma unroll
    for (int j = 0; j < kCopyUnroll; ++j) {
      const unsigned int e = c0 + j * kCopyThreads;
      at[j] = -1;
      if (e < a.piece) {
        at[j] = e;
        if (a.run != a.piece) {
          const unsigned int q = e / a.run, o = q / a.inner;
          at[j] = o * a.outer_stride + (q - o * a.inner) * a.inner_stride + (e - q * a.run);
        }
        x[j] = from[at[j]];
      }
    }
#pragma unroll
    for (int j = 0; j < kCopyUnroll; ++j)
      if (at[j] >= 0) to[at[j]] = x[j];
  }
  if (a.table) {
    const int live = *a.n_live;
    for (long long e = (long long)blockIdx.x * kCopyThreads + threadIdx.x; e < a.entries; e += (long long)gridDim.x * kCopyThreads) {
      const int p = a.table[e];
      if (p >= live && p < a.n_pages) a.table[e] = a.place[p];
    }
  }
}

// most: pages that may have to be copied (how many are is known on the device).
cudaError_t launch_copy(const fc_pages &p, CopyArgs a, long long most, cudaStream_t st) {
  const int per = p.dtype == FC_F32 ? 4 : 8;                           // elements in 16 bytes
  a.k = (uint4 *)p.k; a.v = (uint4 *)p.v;
  a.layer_stride = p.layer_stride / per; a.page_stride = p.page_stride / per; a.n_layers = p.n_layers; a.n_pages = p.n_pages;
  const long long row = p.head_dim / per, hs = p.head_stride / per, ss = p.slot_stride / per;
  a.piece = (unsigned int)(row * p.n_kv_heads * p.page_size);
  // the dimension with the smaller stride inside; dimensions of one entry have none
  const bool slots_inside = p.n_kv_heads == 1 || (p.page_size > 1 && ss <= hs);
  long long inner = slots_inside ? p.page_size : p.n_kv_heads;
  const long long outer = slots_inside ? p.n_kv_heads : p.page_size;
  long long is = slots_inside ? ss : hs, os = slots_inside ? hs : ss;
  long long run = row;
  if (inner == 1 || is == run) {                                        // adjacent rows are one run
    run *= inner;
    inner = outer; is = os; os = 0;
    if (inner == 1 || is == run) { run *= inner; inner = 1; is = 0; }
  }
  a.run = (unsigned int)run; a.inner = (unsigned int)inner; a.inner_stride = is; a.outer_stride = os;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  // Blocks: eight pieces of work each where there is much of it, up to 32 per SM, and no more than four per SM where there may be little, because all
  // have to start.  Measured with 8, 16, 32, 64 blocks per SM: 2.2 GB (7B pages) 366, 358, 345, 339 us; 8 MB (1.1B) 6.8, 7.4, 8.6, 11.1.
  // (Streaming loads and stores: 383 with 8.)
  const long long chunk = kCopyThreads * kCopyUnroll, units = most * p.n_layers * 2 * ((a.piece + chunk - 1) / chunk);
  long long blocks = units / 8 < 4 * 148 ? 4 * 148 : units / 8 > 32 * 148 ? 32 * 148 : units / 8;
  if (blocks > units) blocks = units;
  cfg.gridDim = dim3((unsigned)blocks); cfg.blockDim = dim3(kCopyThreads); cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, pages_copy_kernel, a);
}

// ------------------------------------------------------------------------------------------------ arguments
constexpr size_t kScratchAlign = 256;
size_t aligned(size_t v) { return (v + kScratchAlign - 1) / kScratchAlign * kScratchAlign; }

int table_ok(const void *table, int width, int n_seqs, int page_size) {
  if (!table || width < 1 || n_seqs < 1 || page_size < 1) return FC_ERR_ARG;
  return (long long)width * page_size > INT_MAX - 1024 ? FC_ERR_CAPACITY : FC_OK;
}

// Marks of the table rows named so far; false for one out of range or named twice.
struct Marks {
  unsigned char *m; int n;
  explicit Marks(int rows) : m(new (std::nothrow) unsigned char[rows]), n(rows) { if (m) memset(m, 0, rows); }
  ~Marks() { delete[] m; }
  bool once(int i) { if (i < 0 || i >= n || m[i]) return false; m[i] = 1; return true; }
};

// n named rows, a launch for every list that they fill.
template <typename F>
int by_lists(int n, F launch) {
  for (int i0 = 0; i0 < n; i0 += kListed) {
    const int count = n - i0 < kListed ? n - i0 : kListed;
    if (count <= kFew) { SeqList<kFew> list; launch(list, i0, count); }
    else { SeqList<kListed> list; launch(list, i0, count); }
    if (cudaGetLastError() != cudaSuccess) return FC_ERR_CUDA;
  }
  return FC_OK;
}

}  // namespace

// FC_OK, or why a pool cannot be used.  Rows must not overlap: with the dimensions sorted by stride, each has to reach beyond what lies inside.
int pages_ok(const fc_pages *p) {
  if (!p || !p->k || !p->v || p->k == p->v) return FC_ERR_ARG;
  if (p->dtype != FC_F32 && p->dtype != FC_BF16) return FC_ERR_ARG;
  if (p->n_layers < 1 || p->n_pages < 1 || p->n_kv_heads < 1 || p->page_size < 1) return FC_ERR_ARG;
  if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128) return FC_ERR_SHAPE;
  if (page_too_large(p->n_kv_heads, p->page_size, p->head_dim)) return FC_ERR_CAPACITY;
  const int per = p->dtype == FC_F32 ? 4 : 8;
  if (((uintptr_t)p->k | (uintptr_t)p->v) % 16) return FC_ERR_ARG;
  long long count[4] = {p->n_layers, p->n_pages, p->n_kv_heads, p->page_size};
  long long stride[4] = {p->layer_stride, p->page_stride, p->head_stride, p->slot_stride};
  long long extent = p->head_dim;
  bool done[4] = {count[0] == 1, count[1] == 1, count[2] == 1, count[3] == 1};
  for (int i = 0; i < 4; ++i) {
    int best = -1;
    for (int d = 0; d < 4; ++d)
      if (!done[d] && (best < 0 || stride[d] < stride[best])) best = d;
    if (best < 0) break;
    if (stride[best] % per || stride[best] < extent || stride[best] > (1ll << 46) / count[best]) return FC_ERR_ARG;
    extent += stride[best] * (count[best] - 1);
    done[best] = true;
  }
  return FC_OK;
}

}  // namespace fc

using namespace fc;

extern "C" int fc_op_pages_free(int32_t *table, int32_t table_width, int32_t n_seqs, int32_t *kv_len, int32_t *refs, int32_t n_pages,
                                int32_t page_size, const int32_t *seqs, int32_t n, int32_t window, int32_t n_sink, void *cuda_stream) {
  if (!kv_len || !refs || n_pages < 1 || n < 0 || (n > 0 && !seqs) || window < 0 || n_sink < 0) return FC_ERR_ARG;
  if (int rc = table_ok(table, table_width, n_seqs, page_size)) return rc;
  Marks marks(n_seqs);
  if (!marks.m) return FC_ERR_ARG;
  for (int i = 0; i < n; ++i)
    if (!marks.once(seqs[i])) return FC_ERR_ARG;
  return by_lists(n, [&](auto &list, int i0, int count) {
    memcpy(list.a, seqs + i0, count * sizeof(int));
    pages_free_kernel<<<count, 128, 0, (cudaStream_t)cuda_stream>>>(table, table_width, kv_len, refs, n_pages, page_size, list, window, n_sink);
  });
}

extern "C" int fc_op_pages_fork(int32_t *table, int32_t table_width, int32_t n_seqs, int32_t *kv_len, int32_t *refs, int32_t n_pages,
                                int32_t page_size, const int32_t *src, const int32_t *dst, int32_t n, void *cuda_stream) {
  if (!kv_len || !refs || n_pages < 1 || n < 0 || (n > 0 && (!src || !dst))) return FC_ERR_ARG;
  if (int rc = table_ok(table, table_width, n_seqs, page_size)) return rc;
  Marks marks(n_seqs);
  if (!marks.m) return FC_ERR_ARG;
  for (int i = 0; i < n; ++i)
    if (!marks.once(dst[i])) return FC_ERR_ARG;
  for (int i = 0; i < n; ++i)
    if (src[i] < 0 || src[i] >= n_seqs || marks.m[src[i]]) return FC_ERR_ARG;
  return by_lists(n, [&](auto &list, int i0, int count) {
    memcpy(list.a, src + i0, count * sizeof(int));
    memcpy(list.b, dst + i0, count * sizeof(int));
    pages_fork_kernel<<<count, 128, 0, (cudaStream_t)cuda_stream>>>(table, table_width, kv_len, refs, n_pages, page_size, list);
  });
}

// Scratch of a reservation: three lists of pages, a list of copies, two of sequences, the number of copies.
extern "C" size_t fc_op_pages_reserve_scratch_bytes(int32_t n_pages, int32_t n_seqs) {
  if (n_pages < 1 || n_seqs < 1) return 0;
  return aligned((3 * (size_t)n_pages + 4 * (size_t)n_seqs + 1) * sizeof(int32_t));
}

extern "C" int fc_op_pages_reserve(const fc_pages *pages, int32_t *table, int32_t table_width, int32_t n_seqs, const int32_t *kv_len,
                                   int32_t *refs, int32_t rows, int32_t *served, void *scratch, size_t scratch_bytes, void *cuda_stream) {
  if (int rc = pages_ok(pages)) return rc;
  if (!kv_len || !refs || !scratch || rows < 1 || rows > 64 || (uintptr_t)scratch % kScratchAlign) return FC_ERR_ARG;
  if (int rc = table_ok(table, table_width, n_seqs, pages->page_size)) return rc;
  if (scratch_bytes < fc_op_pages_reserve_scratch_bytes(pages->n_pages, n_seqs)) return FC_ERR_CAPACITY;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  int32_t *s = (int32_t *)scratch;
  ReserveArgs a; memset(&a, 0, sizeof a);
  a.table = table; a.width = table_width; a.n_seqs = n_seqs; a.kv_len = kv_len; a.refs = refs; a.n_pages = pages->n_pages;
  a.page_size = pages->page_size; a.rows = rows; a.served = served;
  a.writers = s; a.keeper = s + a.n_pages; a.free_list = s + 2 * (size_t)a.n_pages;         // behind the free pages: sources and targets of the copies
  a.src = a.free_list + a.n_pages + 2 * (size_t)n_seqs; a.dst = a.src + n_seqs; a.n_copies = a.dst + n_seqs;
  pages_reserve_kernel<<<1, kPlanThreads, 0, st>>>(a);
  if (cudaGetLastError() != cudaSuccess) return FC_ERR_CUDA;
  CopyArgs c; memset(&c, 0, sizeof c);
  c.src = a.free_list + a.n_pages; c.dst = c.src + n_seqs; c.n = a.n_copies;
  return launch_copy(*pages, c, n_seqs, st) == cudaSuccess ? FC_OK : FC_ERR_CUDA;
}

extern "C" size_t fc_op_pages_compact_scratch_bytes(int32_t n_pages) {
  return n_pages < 1 ? 0 : aligned((3 * (size_t)n_pages + 2) * sizeof(int32_t));
}

extern "C" int fc_op_pages_compact(const fc_pages *pages, int32_t *table, int32_t table_width, int32_t n_seqs, int32_t *refs,
                                   int32_t *n_live, void *scratch, size_t scratch_bytes, void *cuda_stream) {
  if (int rc = pages_ok(pages)) return rc;
  if (!refs || !scratch || (uintptr_t)scratch % kScratchAlign) return FC_ERR_ARG;
  if (int rc = table_ok(table, table_width, n_seqs, pages->page_size)) return rc;
  if (scratch_bytes < fc_op_pages_compact_scratch_bytes(pages->n_pages)) return FC_ERR_CAPACITY;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const size_t n = pages->n_pages;
  int32_t *s = (int32_t *)scratch;
  CompactArgs a;
  a.refs = refs; a.n_pages = pages->n_pages; a.dst = s; a.src = s + n; a.place = s + 2 * n; a.counts = s + 3 * n; a.n_live = n_live;
  pages_compact_kernel<<<1, kPlanThreads, 0, st>>>(a);
  if (cudaGetLastError() != cudaSuccess) return FC_ERR_CUDA;
  CopyArgs c; memset(&c, 0, sizeof c);
  c.src = a.src; c.dst = a.dst; c.n = a.counts; c.table = table; c.entries = (long long)table_width * n_seqs; c.place = a.place; c.n_live = a.counts + 1;
  return launch_copy(*pages, c, (pages->n_pages + 1) / 2, st) == cudaSuccess ? FC_OK : FC_ERR_CUDA;
}
