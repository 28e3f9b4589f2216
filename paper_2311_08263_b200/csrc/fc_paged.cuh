// Attention over pages: the line of key tiles that CTAs share, and joining the parts of a unit (k_paged_attn.cu, k_paged_umma.cu).
#pragma once
#include <cstring>

#include "fc_attn.cuh"
#include "fc_internal.h"
#include "fc_paged.h"
#include "fc_ptx.cuh"

namespace fc {

namespace {

constexpr int kWorkers = 148;          // CTAs on the line: one per SM

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

// Tiles of the whole call, and of the sequences in front of sequence `upto` (a warp does this together).
template <int KEYS>
__device__ __forceinline__ void count_tiles(const PagedAttnArgs &a, int upto, long long &total, long long &before) {
  const int lane = threadIdx.x & 31, units = a.groups * a.pool.n_kv_heads;
  long long all = 0, some = 0;
  for (int b = lane; b < a.batch; b += 32) {
    int len;
    const long long n = (long long)seq_tiles<KEYS>(a, b, len).n * units;
    all += n;
    if (b < upto) some += n;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    all += __shfl_xor_sync(0xffffffffu, all, o);
    some += __shfl_xor_sync(0xffffffffu, some, o);
  }
  total = all;
  before = some;
}
// The place of tile f of the line (a warp together; f is inside the line).
template <int KEYS>
__device__ __forceinline__ Place find_place(const PagedAttnArgs &a, long long f) {
  const int lane = threadIdx.x & 31, units = a.groups * a.pool.n_kv_heads;
  long long base = 0;
  Place p = {0, 0, 0, 0, -1, {0, 0, 0}};
  for (int b0 = 0; b0 < a.batch; b0 += 32) {
    int len = -1;
    KeyTiles k = {0, 0, 0};
    if (b0 + lane < a.batch) k = seq_tiles<KEYS>(a, b0 + lane, len);
    long long x = (long long)k.n * units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    const unsigned int beyond = __ballot_sync(0xffffffffu, base + x > f);
    if (beyond) {
      const int w = __ffs(beyond) - 1;
      p.k.n = __shfl_sync(0xffffffffu, k.n, w);
      p.k.sinks = __shfl_sync(0xffffffffu, k.sinks, w);
      p.k.first = __shfl_sync(0xffffffffu, k.first, w);
      p.len = __shfl_sync(0xffffffffu, len, w);
      p.b = b0 + w;
      const long long at = f - (base + __shfl_sync(0xffffffffu, x, w) - (long long)p.k.n * units);
      const int u = (int)(at / p.k.n);
      p.t = (int)(at - (long long)u * p.k.n);
      p.kvh = u / a.groups;
      p.qg = u - p.kvh * a.groups;
      return p;
    }
    base += __shfl_sync(0xffffffffu, x, 31);
  }
  return p;
}

// Result of a query: un-normalised sums over `den`.  A row that sees nothing is 0, one beyond the table NaN.
__device__ __forceinline__ float result_scale(const PagedAttnArgs &a, int pos, float den) {
  return pos >= a.cap ? quiet_nan() : den == 0.f ? 0.f : 1.0f / den;
}

// ------------------------------------------------------------------------------------ joining the parts of a unit
// A block takes block_rows queries of a unit: with items = queries x hd / 4 pieces of four elements, threads are groups that take turns at the
// parts.  A few units have many parts each (one sequence, four kv heads: 37), and then a query per block reads them all at once.
constexpr int kCombine = 256;

template <int HD, int Q, int KEYS>
__global__ void __launch_bounds__(kCombine) paged_combine_kernel(const __grid_constant__ PagedAttnArgs a, int workers, int block_rows) {
  __shared__ long long counts[2];
  __shared__ float4 acc_s[kCombine];
  __shared__ float2 ml_s[kCombine];
  const int units = a.groups * a.pool.n_kv_heads, b = blockIdx.x / units, u = blockIdx.x - b * units, tid = threadIdx.x;
  int len;
  const KeyTiles k = seq_tiles<KEYS>(a, b, len);
  if (tid < 32) {
    long long total, before;
    count_tiles<KEYS>(a, b, total, before);
    if (tid == 0) { counts[0] = total; counts[1] = before; }
  }
  __syncthreads();
  const int group = a.hq / a.pool.n_kv_heads, nq = group * a.c;
  const int kvh = u / a.groups, q0 = (u - kvh * a.groups) * Q, row0 = blockIdx.y * block_rows;
  const int n_rows = min(block_rows, min(Q, nq - q0) - row0), items = n_rows * (HD / 4);
  if (n_rows <= 0) return;
  const long long chunk = chunk_of(counts[0], workers), begin = counts[1] + (long long)u * k.n;
  UnitParts w = {0, -1};
  if (k.n > 0) {
    w = unit_parts(begin, k.n, chunk);
    if (w.first == w.last && !a.status) return;          // written by its one CTA
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  bool lost = false;                                     // a CTA that gave up a wait left nothing that counts
  if (a.status) {
    for (int i = w.first; i <= w.last; ++i) lost |= __ldcg(a.status + i) != 0u;
    if (w.first == w.last && !lost) return;
  }
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
      constexpr int U = 4;
      for (int p = w.first + g; p <= w.last; p += groups * U) {
        float2 v[U];
        float4 x[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int at = p + i * groups;
          v[i] = make_float2(-INFINITY, 0.f);
          x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (at <= w.last) {
            const float *part = a.parts + ((long long)at * 2 + part_place(begin, at, chunk)) * (Q * (HD + 2));
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
      const int q = q0 + row0 + row, j = q / group, h = kvh * group + q - j * group;
      const float f = lost ? quiet_nan() : len < 0 ? 0.f : result_scale(a, len + j, den);
      *reinterpret_cast<float4 *>(a.out + (((long long)b * a.c + j) * a.hq + h) * HD + c4 * 4) = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
    }
  }
}

// Blocks of the launch behind a line of `workers` CTAs: whole units, or fewer queries per block while there are not enough blocks for the GPU.
template <int HD, int Q, int KEYS>
cudaError_t launch_combine(const PagedAttnArgs &a, int workers, cudaStream_t st) {
  const long long units = (long long)a.batch * a.groups * a.pool.n_kv_heads;
  int rows = Q < 16 ? Q : 16;
  while (rows > 1 && units * (Q / rows) < workers) rows /= 2;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3((unsigned)units, Q / rows); cfg.blockDim = dim3(kCombine); cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, paged_combine_kernel<HD, Q, KEYS>, a, workers, rows);
}
template <typename K>
cudaError_t allow_smem(K kernel, size_t bytes, bool *done) {
  const int dev = current_device_slot();
  if (done[dev]) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  done[dev] = e == cudaSuccess;
  return e;
}

}  // namespace
}  // namespace fc
