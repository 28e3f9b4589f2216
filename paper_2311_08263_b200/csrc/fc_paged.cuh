// Attention over pages: the line of key tiles that CTAs share, and joining the parts of a unit (k_paged_attn.cu, k_paged_umma.cu).
#pragma once
#include <cstring>

#include "fc_attn.cuh"
#include "fc_internal.h"
#include "fc_paged.h"
#include "fc_ptx.cuh"

namespace fc {

namespace {

constexpr int kSms = kPagedSms;        // CTAs on the line: one per SM

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// What a part with maximum m and sum l counts against a maximum M; one that saw nothing counts nothing.
__device__ __forceinline__ float part_weight(float2 part, float M, float sl2) {
  return part.x == -INFINITY && part.y == 0.f ? 0.f : ex2((part.x - M) * sl2);
}
__device__ __forceinline__ float quiet_nan() { return __int_as_float(0x7fffffff); }

template <int KEYS>
__device__ __forceinline__ KeyTiles seq_tiles(const PagedAttnArgs &a, int b, int &len) {
  len = clamp_len(a.kv_len[b], a.cap);
  return key_tiles(len, a.c, a.cap, a.window, a.n_sink, KEYS);
}

// A place on the line of tiles: tile t of a unit (kv head, group of queries) of sequence b.
struct Place {
  int b, kvh, qg, t, len;
  KeyTiles k;
};
// `step` tiles on; returns how many units that is.
template <int KEYS>
__device__ __forceinline__ int move_on(const PagedAttnArgs &a, Place &p, int step) {
  int units = 0;
  p.t += step;
  while (p.t >= p.k.n) {
    p.t -= p.k.n;
    ++units;
    if (++p.qg == a.groups) {
      p.qg = 0;
      if (++p.kvh == a.pool.n_kv_heads) {
        p.kvh = 0;
        do {
          if (++p.b >= a.batch) { p.k.n = 0x7fffffff; return units; }      // behind the line: nobody asks
          p.k = seq_tiles<KEYS>(a, p.b, p.len);
        } while (p.k.n == 0);
      }
    }
  }
  return units;
}

// Sum over a warp, to all lanes.
__device__ __forceinline__ int warp_sum_i(int v) { return __reduce_add_sync(0xffffffffu, v); }

// Tiles of the whole line, and of the sequences in front of sequence `upto` (a warp does this together).
template <int KEYS>
__device__ __forceinline__ void count_tiles(const PagedAttnArgs &a, int upto, int &total, int &before) {
  const int lane = threadIdx.x & 31, units = a.groups * a.pool.n_kv_heads;
  int all = 0, some = 0;
#pragma unroll 1
  for (int b = lane; b < a.batch; b += 32) {
    int len;
    const int n = seq_tiles<KEYS>(a, b, len).n * units;
    all += n;
    if (b < upto) some += n;
  }
  total = warp_sum_i(all);
  before = warp_sum_i(some);
}
// The place of tile f of the line (a warp together; f is inside the line).
template <int KEYS>
__device__ __forceinline__ Place find_place(const PagedAttnArgs &a, int f) {
  const int lane = threadIdx.x & 31, units = a.groups * a.pool.n_kv_heads;
  Place p = {0, 0, 0, 0, -1, {0, 0, 0}};
#pragma unroll 1
  for (int b0 = 0; b0 < a.batch; b0 += 32) {
    int len = -1;
    KeyTiles k = {0, 0, 0};
    if (b0 + lane < a.batch) k = seq_tiles<KEYS>(a, b0 + lane, len);
    int x = k.n * units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    const unsigned int beyond = __ballot_sync(0xffffffffu, x > f);
    if (beyond) {
      const int w = __ffs(beyond) - 1;
      p.k.n = __shfl_sync(0xffffffffu, k.n, w);
      p.k.sinks = __shfl_sync(0xffffffffu, k.sinks, w);
      p.k.first = __shfl_sync(0xffffffffu, k.first, w);
      p.len = __shfl_sync(0xffffffffu, len, w);
      p.b = b0 + w;
      const int at = f - (__shfl_sync(0xffffffffu, x, w) - p.k.n * units);
      const int u = (int)((unsigned int)at / (unsigned int)p.k.n);
      p.t = at - u * p.k.n;
      p.kvh = (int)((unsigned int)u / (unsigned int)a.groups);
      p.qg = u - p.kvh * a.groups;
      return p;
    }
    f -= __shfl_sync(0xffffffffu, x, 31);
  }
  return p;
}

// Result of a query: un-normalised sums over `den`.  A row beyond the table is NaN, and so is one whose scores are all minus infinity (zeros over zero).
__device__ __forceinline__ float result_scale(const PagedAttnArgs &a, int pos, float den) {
  return pos >= a.cap ? quiet_nan() : 1.0f / den;
}

// Byte offset of 16-byte piece `ch` of key `r` in a tile of KEYS rows of ROW bytes: sub-tiles of 128 bytes a row, pieces permuted so that eight rows at
// one piece lie in different banks.
template <int KEYS, int ROW>
__device__ __forceinline__ uint32_t poff(int r, int ch) {
  if (ROW == 64) return (uint32_t)r * 64u + (uint32_t)((ch ^ ((r >> 1) & 3)) << 4);
  return (uint32_t)(ch >> 3) * (KEYS * 128u) + (uint32_t)r * 128u + (uint32_t)(((ch & 7) ^ (r & 7)) << 4);
}

// A warp's own stream of tiles: those of its piece of the line, or every WARPS-th of its CTA's in a cluster, into a ring of S stages (keys, then values, of KEYS rows of ROW bytes).
// The lanes' keys are looked up in the table a tile ahead of the copies, which first use what was read then.
template <int KEYS, int ROW, int S, int QUERIES, bool LINE, int WARPS>
struct TileStream {
  static constexpr uint32_t kHalf = KEYS * ROW, kTile = 2 * kHalf;
  static constexpr int STEP = LINE ? 1 : WARPS;
  static constexpr int PER = ROW / 16, RPI = 32 / PER;   // 16-byte pieces of a row; rows that the lanes load at once
  static constexpr int kUnseen = -2;                     // a key that no query sees; -1: the table has no page for it
  static_assert(KEYS <= 32 && 32 % KEYS == 0 && KEYS % RPI == 0, "lanes, keys and rows");
  const PagedAttnArgs &a;
  Place at;
  int i, n, nq;                                          // next tile, tiles of the piece; queries of a kv head
  int see_from, see_to;                                  // keys that some query of the unit sees: the sinks, and from .. to
  int page, slot;
  uint32_t ring;                                         // shared memory
  unsigned int *bad_keys;                                // [S] keys of a tile whose page is missing

  __device__ __forceinline__ TileStream(const PagedAttnArgs &args, const Place &begin, int first, int count, uint32_t smem, unsigned int *bad)
      : a(args), at(begin), i(first), n(count), page(kUnseen), slot(0), ring(smem), bad_keys(bad) {
    nq = a.nq;
    if (i < n) {
      at.t += first;                                     // in a cluster: tiles of one unit
      unit_keys();
      look_up();
    }
  }
  __device__ __forceinline__ void unit_keys() {
    see_from = window_first(at.len + quotient16(at.qg * QUERIES, a.group_inv), a.window);          // the first row's window reaches furthest back
    see_to = min(at.len + quotient16(min(nq - 1, at.qg * QUERIES + QUERIES - 1), a.group_inv), a.cap - 1);
  }
  __device__ __forceinline__ void look_up() {
    const int t = tile_key(at.k, at.t, KEYS) + (threadIdx.x & (KEYS - 1));
    page = kUnseen;
    if (t <= see_to && (t >= see_from || t < a.n_sink)) {
      const int e = (int)((unsigned int)t / (unsigned int)a.pool.page_size);
      slot = t - e * a.pool.page_size;
      page = max(-1, a.table[(long long)at.b * a.width + e]);
    }
  }
  // Copies of the next tile (or of nothing) into a stage, as one group.
  __device__ __forceinline__ void request(int stage) {
    if (i < n) {
      const int lane = threadIdx.x & 31;
      const bool there = page >= 0 && page < a.pool.n_pages;
      const unsigned int bad = __ballot_sync(0xffffffffu, !there && page != kUnseen);
      if (lane == 0) bad_keys[stage] = bad;              // (KEYS < 32: the lanes hold the keys several times)
      const long long off = there ? (long long)page * a.page_bytes + (long long)slot * a.slot_bytes : -1;
      const uint32_t kb = ring + stage * kTile;
      const char *k0 = (const char *)a.pool.k + at.kvh * a.head_bytes + (lane % PER) * 16;
      const char *v0 = (const char *)a.pool.v + at.kvh * a.head_bytes + (lane % PER) * 16;
#pragma unroll
      for (int y = 0; y < KEYS / RPI; ++y) {
        const int r = y * RPI + lane / PER;
        const long long o = __shfl_sync(0xffffffffu, off, r);
        const uint32_t d = kb + poff<KEYS, ROW>(r, lane % PER), bytes = o < 0 ? 0u : 16u;      // keys that no row sees become zeros
        copy16(d, k0 + (o < 0 ? 0 : o), bytes);
        copy16(d + kHalf, v0 + (o < 0 ? 0 : o), bytes);
      }
      i += STEP;
      if (i < n) {
        if (LINE) {
          if (move_on<KEYS>(a, at, STEP)) unit_keys();
        } else {
          at.t += STEP;
        }
        look_up();
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
};

// What there is to do: the place of the first tile, and how many.  LINE: a worker's piece of the line; else a CTA's share of one unit (grid: CTAs of the
// cluster, units, sequences).  False where the line has nothing for the worker.
template <int KEYS, bool LINE>
__device__ __forceinline__ bool my_piece(const PagedAttnArgs &a, int worker, int workers, Place &seg, int &n) {
  if (LINE) {
    int total, unused;
    count_tiles<KEYS>(a, 0, total, unused);
    const int chunk = chunk_of(total, workers), f0 = chunk * worker;       // chunk x workers < 2^31 + workers
    if (f0 >= total || f0 < 0) return false;
    n = min(total - f0, chunk);
    seg = find_place<KEYS>(a, f0);
  } else {
    seg.b = blockIdx.z; seg.kvh = blockIdx.y / a.groups; seg.qg = blockIdx.y - seg.kvh * a.groups;
    seg.k = seq_tiles<KEYS>(a, seg.b, seg.len);
    const int cut = (seg.k.n + gridDim.x - 1) / gridDim.x;
    seg.t = cut * blockIdx.x;
    n = max(0, min(cut, seg.k.n - seg.t));
  }
  return true;
}

// The parts of a cluster: un-normalised sums [rows][HD] at `sums` and (max, sum) at `ml` in each CTA's shared memory.  Every CTA writes a share of the rows.
template <int HD>
__device__ __forceinline__ void join_cluster(const PagedAttnArgs &a, const Place &seg, int q0, int rows, uint32_t sums, uint32_t ml, int threads) {
  const int ns = gridDim.x, group = a.group;
  const float sl2 = rsqrtf((float)HD) * 1.4426950408889634f;
  cluster_sync_all();
  for (int e = blockIdx.x * threads + threadIdx.x; e < rows * (HD / 4); e += ns * threads) {
    const int row = e / (HD / 4), c4 = e - row * (HD / 4);
    float2 mv[8];
    float4 ov[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      mv[r] = make_float2(-INFINITY, 0.f);
      ov[r] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < ns) {
        mv[r] = ld_cluster_f2(map_to_cta(ml + (uint32_t)row * 8u, (uint32_t)r));
        ov[r] = ld_cluster_f4(map_to_cta(sums + (uint32_t)(row * HD + c4 * 4) * 4u, (uint32_t)r));
      }
    }
    float M = -INFINITY, den = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int r = 0; r < 8; ++r) M = fmaxf(M, mv[r].x);
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const float f = part_weight(mv[r], M, sl2);
      den = fmaf(mv[r].y, f, den);
      acc.x = fmaf(f, ov[r].x, acc.x); acc.y = fmaf(f, ov[r].y, acc.y); acc.z = fmaf(f, ov[r].z, acc.z); acc.w = fmaf(f, ov[r].w, acc.w);
    }
    const int q = q0 + row, j = quotient16(q, a.group_inv), h = seg.kvh * group + q - j * group;
    const float f = seg.len < 0 ? 0.f : result_scale(a, seg.len + j, den);
    *reinterpret_cast<float4 *>(a.out + (((long long)seg.b * a.c + j) * a.hq + h) * HD + c4 * 4) = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
  }
  cluster_sync_all();                                    // the others may still be reading this CTA's memory
}

// ------------------------------------------------------------------------------------ joining the parts of a unit
// A block takes block_rows queries of a unit: with items = queries x hd / 4 pieces of four elements, threads are groups that take turns at the
// parts.  A few units have many parts each (one sequence, four kv heads, 32000 keys: some 290), and then a query per block reads them all at once.

constexpr int kCombine = 256;
// U: parts that a thread has on their way at once.
template <int HD, int Q, int KEYS, int U>
__global__ void __launch_bounds__(kCombine) paged_combine_kernel(const __grid_constant__ PagedAttnArgs a, int workers, int block_rows) {
  __shared__ int counts[2];
  __shared__ float4 acc_s[kCombine];
  __shared__ float2 ml_s[kCombine];
  const int units = a.groups * a.pool.n_kv_heads, b = blockIdx.x / units, u = blockIdx.x - b * units, tid = threadIdx.x;
  int len;
  const KeyTiles k = seq_tiles<KEYS>(a, b, len);
  if (tid < 32) {
    int total, before;
    count_tiles<KEYS>(a, b, total, before);
    if (tid == 0) { counts[0] = total; counts[1] = before; }
  }
  __syncthreads();
  const int group = a.group, nq = a.nq;
  const int kvh = u / a.groups, q0 = (u - kvh * a.groups) * Q, row0 = blockIdx.y * block_rows;
  const int n_rows = min(block_rows, min(Q, nq - q0) - row0), items = n_rows * (HD / 4);
  if (n_rows <= 0) return;
  const int chunk = chunk_of(counts[0], workers), begin = counts[1] + u * k.n;
  UnitParts w = {0, -1};
  if (k.n > 0) {
    w = unit_parts(begin, k.n, chunk);
    // written by its one worker; but one block always waits, so that this kernel does not end before the line does
    if (w.first == w.last && !a.status && (blockIdx.x | blockIdx.y)) return;
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  bool lost = false;                                     // a CTA that gave up a wait left nothing that counts
  if (a.status) lost = __syncthreads_or(tid <= w.last - w.first && __ldcg(a.status + w.first + tid) != 0u);
  if (w.first == w.last && !lost) return;
  const float sl2 = rsqrtf((float)HD) * 1.4426950408889634f;
  int groups = 1;
  while (groups * 2 * items <= kCombine) groups *= 2;
  const int g = items <= kCombine ? tid / items : 0;
  for (int e0 = 0; e0 < items; e0 += kCombine) {
    const int e = items <= kCombine ? tid - g * items : e0 + tid;
    const int row = e / (HD / 4), c4 = e - row * (HD / 4);
    float m = -INFINITY, den = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (e < items && g < groups) {
      for (int p = w.first + g; p <= w.last; p += groups * U) {
        float2 v[U];
        float4 x[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int at = p + i * groups;
          v[i] = make_float2(-INFINITY, 0.f);
          x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (at <= w.last) {
            const float *part = a.parts + ((long long)at * 2 + part_place(begin, at, chunk)) * part_floats(Q, HD);
            v[i] = __ldcg(reinterpret_cast<const float2 *>(part + Q * HD + (row0 + row) * 2));
            x[i] = __ldcg(reinterpret_cast<const float4 *>(part + (row0 + row) * HD + c4 * 4));
          }
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < U; ++i) top = fmaxf(top, v[i].x);
        const float f = m == top ? 1.f : ex2((m - top) * sl2);
        m = top;
        den *= f; acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const float s = part_weight(v[i], top, sl2);
          den = fmaf(v[i].y, s, den);
          acc.x = fmaf(s, x[i].x, acc.x); acc.y = fmaf(s, x[i].y, acc.y); acc.z = fmaf(s, x[i].z, acc.z); acc.w = fmaf(s, x[i].w, acc.w);
        }
      }
    }
    if (groups > 1) {
      acc_s[tid] = acc;
      ml_s[tid] = make_float2(m, den);
      __syncthreads();
      if (g == 0) {
        float top = m;
        for (int i = 1; i < groups; ++i) top = fmaxf(top, ml_s[tid + i * items].x);
        float f = part_weight(make_float2(m, den), top, sl2);
        den *= f; acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
        for (int i = 1; i < groups; ++i) {
          const float2 v = ml_s[tid + i * items];
          const float4 x = acc_s[tid + i * items];
          f = part_weight(v, top, sl2);
          den = fmaf(v.y, f, den);
          acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
        }
      }
    }
    if (e < items && g == 0) {
      const int q = q0 + row0 + row, j = quotient16(q, a.group_inv), h = kvh * group + q - j * group;
      const float f = lost ? quiet_nan() : len < 0 ? 0.f : result_scale(a, len + j, den);
      *reinterpret_cast<float4 *>(a.out + (((long long)b * a.c + j) * a.hq + h) * HD + c4 * 4) = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
    }
  }
}

// Blocks of the launch behind the line: whole units, or fewer queries per block while there are not enough blocks for the GPU.
template <int HD, int Q, int KEYS>
cudaError_t launch_combine(const PagedAttnArgs &a, int workers, cudaStream_t st) {
  const long long units = (long long)a.batch * a.groups * a.pool.n_kv_heads;
  int rows = Q < 16 ? Q : 16;
  while (rows > 1 && units * (Q / rows) < kSms) rows /= 2;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3((unsigned)units, Q / rows); cfg.blockDim = dim3(kCombine); cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, rows == 1 ? paged_combine_kernel<HD, Q, KEYS, 8> : paged_combine_kernel<HD, Q, KEYS, 4>, a, workers, rows);
}
template <typename K>
cudaError_t allow_smem(K kernel, size_t bytes, bool *done) {
  const int dev = current_device_slot();
  if (done[dev]) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  done[dev] = e == cudaSuccess;
  return e;
}

// What the kernels know of a call's queries, for units of Q of them.
inline void set_groups(PagedAttnArgs &a, int Q) {
  a.group = a.hq / a.pool.n_kv_heads;
  a.nq = a.group * a.c;
  a.groups = (a.nq + Q - 1) / Q;
  a.group_inv = reciprocal16(a.group);
}
// A launch for as many sequences at a time as a line can hold (all of them, but for tables of billions of positions).
template <typename F>
cudaError_t by_lines(const PagedAttnArgs &all, int keys, F launch) {
  const int most = line_batch(all.groups * all.pool.n_kv_heads, all.cap, keys);
  if (most == 0) return cudaErrorInvalidValue;
  for (int b0 = 0; b0 < all.batch; b0 += most) {
    PagedAttnArgs a = all;
    a.batch = all.batch - b0 < most ? all.batch - b0 : most;
    a.table += (long long)b0 * a.width;
    a.kv_len += b0;
    a.first = b0;
    a.q = (const char *)a.q + (long long)b0 * a.c * a.q_stride * a.elem_bytes;
    a.out += (long long)b0 * a.c * a.hq * all.hd;
    if (cudaError_t e = launch(a)) return e;
  }
  return cudaSuccess;
}

// The line, a piece for every warp, and the kernel that joins its parts.
template <int HD, int Q, int KEYS, typename K>
cudaError_t launch_line(PagedAttnArgs a, const PagedPlan &plan, K line, size_t smem, bool *done, cudaStream_t st) {
  if (plan.queries != Q || plan.keys != KEYS) return cudaErrorInvalidValue;
  set_groups(a, Q);
  if (cudaError_t e = allow_smem(line, smem, done)) return e;
  return by_lines(a, KEYS, [&](const PagedAttnArgs &part) {
    line<<<kSms, plan.workers / kSms * 32, smem, st>>>(part);
    if (cudaError_t e = cudaGetLastError()) return e;
    return launch_combine<HD, Q, KEYS>(part, plan.workers, st);
  });
}
// The same, or clusters where the plan says so.
template <int HD, int Q, int KEYS, typename K>
cudaError_t launch_units(PagedAttnArgs a, const PagedPlan &plan, K line, K cluster, size_t smem, bool (*done)[kMaxDevices], cudaStream_t st) {
  if (plan.ctas == 0) return launch_line<HD, Q, KEYS>(a, plan, line, smem, done[0], st);
  if (plan.queries != Q || plan.keys != KEYS) return cudaErrorInvalidValue;
  set_groups(a, Q);
  if (cudaError_t e = allow_smem(cluster, smem, done[1])) return e;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3(plan.ctas, plan.units, a.batch); cfg.blockDim = dim3(kPagedWarps * 32); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)plan.ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, cluster, a);
}

}  // namespace
}  // namespace fc
