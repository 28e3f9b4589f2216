// Window attention over pages: out = softmax(q.k / sqrt(hd)) v over the keys that a row sees, keys and values behind a table of pages.
//
// paged_mma_kernel (bf16).  One CTA per SM.  The work is a line of key tiles (32 keys), sequence by sequence and unit by unit (a kv head
// and 16 queries: window rows x heads of the group), cut into equal pieces, one per CTA, whatever the lengths of the sequences: the
// launch depends on no length, and a batch of ragged caches is as balanced as one long cache.  The warps of a CTA take turns at its tiles.
// A warp loads its own tiles into its own ring (cp.async, 16 bytes a lane, the lanes look up the pages of the tile's keys), so that it waits for nobody while
// it streams, and the ring runs on across units.  Scores, probabilities and the 16 x hd output stay in its registers; the
// accumulators of Q.K^T are the A operand of P.V as they are.  Where a unit ends (or the CTA's piece), the warps exchange their results through
// shared memory, each adds up a part of the columns, and the unit is written; a unit that several CTAs share goes to scratch as un-normalised parts.
// paged_combine_kernel adds those up in order, and writes the rows that see nothing.
//
// Probabilities enter the tensor cores as three bf16 parts (their sum has all 24 bits), a tile's product is added to the output in fp32: what is rounded
// is what is stored in the cache, nothing else.  (Two parts leave 1.5e-6, relative, of the result.)
#include <cstring>

#include "fc_attn.cuh"
#include "fc_internal.h"
#include "fc_paged.h"
#include "fc_ptx.cuh"

namespace fc {

namespace {

constexpr int kKeys = 32;              // keys per tile

template <int HD>
struct PagedCfg {
  static constexpr int W = HD == 64 ? 8 : 4;                       // warps
  static constexpr int S = HD == 32 ? 8 : 3;                       // stages of a warp's ring
  static constexpr uint32_t kHalf = kKeys * HD * 2, kTile = 2 * kHalf;
  static constexpr int NB = HD / 8, OWN = NB / W;                  // column blocks of the output; of them a warp's own in the exchange
  static constexpr size_t kRing = (size_t)W * S * kTile;
  static constexpr size_t kExchange = (size_t)W * (W - 1) * OWN * 32 * 16;
  static constexpr size_t kSmem = 128 + kRing + kExchange;
};

// Byte offset of 16-byte piece `ch` of key `r` in a tile: rows of 128 bytes (two side by side in sub-tiles at hd 128), pieces
// permuted so that eight rows at one piece lie in different banks.
template <int HD>
__device__ __forceinline__ uint32_t poff(int r, int ch) {
  if (HD == 32) return (uint32_t)r * 64u + (uint32_t)((ch ^ ((r >> 1) & 3)) << 4);
  return (uint32_t)(ch >> 3) * (kKeys * 128u) + (uint32_t)r * 128u + (uint32_t)(((ch & 7) ^ (r & 7)) << 4);
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// Units of a sequence, tiles of a unit, of sequence b.
__device__ __forceinline__ KeyTiles seq_tiles(const PagedAttnArgs &a, int b, int &len) {
  len = clamp_len(a.kv_len[b], a.cap);
  return key_tiles(len, a.c, a.cap, a.window, a.n_sink, kKeys);
}

// A place on the line of tiles: tile t of unit u of sequence b.
struct Place {
  int b, u, t, len;
  KeyTiles k;
};
// The next place `step` tiles on; the caller knows that there is one.
__device__ __forceinline__ void move_on(const PagedAttnArgs &a, Place &p, int step) {
  p.t += step;
  while (p.t >= p.k.n) {
    p.t -= p.k.n;
    if (++p.u == a.units) {
      p.u = 0;
      do {
        if (++p.b >= a.batch) { p.k.n = 0x7fffffff; return; }
        p.k = seq_tiles(a, p.b, p.len);
      } while (p.k.n == 0);
    }
  }
}

// Tiles of the whole call, and of the sequences in front of sequence `upto` (a warp does this together).
__device__ __forceinline__ void count_tiles(const PagedAttnArgs &a, int upto, long long &total, long long &before) {
  const int lane = threadIdx.x & 31;
  long long all = 0, some = 0;
  for (int b = lane; b < a.batch; b += 32) {
    int len;
    const long long n = (long long)seq_tiles(a, b, len).n * a.units;
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
__device__ __forceinline__ Place find_place(const PagedAttnArgs &a, long long f) {
  const int lane = threadIdx.x & 31;
  long long base = 0;
  Place p = {0, 0, 0, -1, {0, 0, 0}};
  for (int b0 = 0; b0 < a.batch; b0 += 32) {
    int len = -1;
    KeyTiles k = {0, 0, 0};
    if (b0 + lane < a.batch) k = seq_tiles(a, b0 + lane, len);
    long long x = (long long)k.n * a.units;
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
      const long long at = f - (base + __shfl_sync(0xffffffffu, x, w) - (long long)p.k.n * a.units);
      p.u = (int)(at / p.k.n);
      p.t = (int)(at - (long long)p.u * p.k.n);
      return p;
    }
    base += __shfl_sync(0xffffffffu, x, 31);
  }
  return p;
}

// Result of a query: un-normalised sums over `den`.  A row that sees nothing is 0, one beyond the table NaN.
__device__ __forceinline__ float result_scale(const PagedAttnArgs &a, int pos, float den) {
  return pos >= a.cap ? __int_as_float(0x7fffffff) : den == 0.f ? 0.f : 1.0f / den;
}

template <int HD>
__global__ void __launch_bounds__(PagedCfg<HD>::W * 32, 1) paged_mma_kernel(const __grid_constant__ PagedAttnArgs a) {
  using C = PagedCfg<HD>;
  constexpr int W = C::W, S = C::S, KS = HD / 16, NT = kKeys / 8, NB = C::NB, OWN = C::OWN;
  constexpr int PER = HD / 8, RPI = 32 / PER;            // 16-byte pieces of a row; rows that the lanes of a warp load at once
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ unsigned char smem_raw[];
  __shared__ float2 ml[W][16];                           // (max, sum) per warp and query
  __shared__ unsigned int bad_keys[W][S];                // keys of a tile whose page is missing

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g4 = lane >> 2, t4 = lane & 3;
  const uint32_t base = (smem_u32(smem_raw) + 127u) & ~127u;
  const uint32_t ring = base + (uint32_t)warp * (S * C::kTile);
  unsigned char *ring_g = smem_raw + (ring - smem_u32(smem_raw));
  float4 *exchange = reinterpret_cast<float4 *>(smem_raw + (base - smem_u32(smem_raw)) + C::kRing);

  long long total, unused;
  count_tiles(a, 0, total, unused);
  const long long chunk = chunk_of(total, gridDim.x), f0 = chunk * blockIdx.x;
  if (f0 >= total) return;
  const int n_mine = (int)(total - f0 < chunk ? total - f0 : chunk);
  Place seg = find_place(a, f0);                         // where the segment (a unit's tiles in this piece) begins
  Place ld = seg;                                        // the tile that is requested next
  if (warp < n_mine && warp > 0) move_on(a, ld, warp);
  int ld_i = warp;
  const int group = a.hq / a.pool.n_kv_heads, nq = group * a.c, nqg = a.units / a.pool.n_kv_heads;
  const float sl2 = rsqrtf((float)HD) * 1.4426950408889634f;

  // the lanes' keys of the next tile: page and offset are looked up a tile ahead of the copies
  int next_key = 0, next_page = -1;
  bool next_seen = false;
  auto look_up = [&]() {
    next_seen = false;
    if (ld_i < n_mine) {
      const int qg = ld.u % nqg;
      const int p_first = ld.len + qg * 16 / group, p_last = ld.len + min(nq - 1, qg * 16 + 15) / group;
      next_key = tile_key(ld.k, ld.t, kKeys) + lane;
      // keys that some row of the unit sees: the first row's window reaches furthest back
      next_seen = next_key <= p_last && (next_key >= window_first(p_first, a.window) || next_key < a.n_sink) && next_key < a.cap;
      if (next_seen) next_page = page_of(a.table + (long long)ld.b * a.width, a.width, next_key, a.pool.page_size, a.pool.n_pages);
    }
  };
  auto request = [&](int stage) {
    if (ld_i < n_mine) {
      const int kvh = ld.u / nqg;
      long long off = -1;
      if (next_seen && next_page >= 0)
        off = (long long)next_page * a.pool.page_stride + (long long)(next_key % a.pool.page_size) * a.pool.slot_stride;
      const unsigned int bad = __ballot_sync(0xffffffffu, next_seen && next_page < 0);
      if (lane == 0) bad_keys[warp][stage] = bad;
      const uint32_t kb = ring + stage * C::kTile;
      const __nv_bfloat16 *k0 = (const __nv_bfloat16 *)a.pool.k + kvh * a.pool.head_stride + (lane % PER) * 8;
      const __nv_bfloat16 *v0 = (const __nv_bfloat16 *)a.pool.v + kvh * a.pool.head_stride + (lane % PER) * 8;
#pragma unroll
      for (int i = 0; i < kKeys / RPI; ++i) {
        const int r = i * RPI + lane / PER;
        const long long o = __shfl_sync(0xffffffffu, off, r);
        const uint32_t d = kb + poff<HD>(r, lane % PER), bytes = o < 0 ? 0u : 16u;      // keys that no row sees become zeros
        copy16(d, k0 + (o < 0 ? 0 : o), bytes);
        copy16(d + C::kHalf, v0 + (o < 0 ? 0 : o), bytes);
      }
      ld_i += W;
      if (ld_i < n_mine) move_on(a, ld, W);
      look_up();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  look_up();
#pragma unroll
  for (int s = 0; s < S - 1; ++s) request(s);

  int stage = 0;
  int i = warp;                                          // this warp's next tile in the piece
  int done = 0;                                          // tiles of the piece in front of the segment
  while (true) {
    // ---- a segment: tiles done .. done + seg_n of the piece, tiles seg.t .. of the unit
    const int seg_n = min(n_mine - done, seg.k.n - seg.t);
    const int kvh = seg.u / nqg, qg = seg.u - kvh * nqg;
    const int q0 = qg * 16, q_last = min(nq - 1, q0 + 15);
    int pos[2], low[2];
    uint32_t qf[KS][4];
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int q = min(q0 + g4 + hh * 8, nq - 1), j = q / group, h = kvh * group + q - j * group;
      pos[hh] = seg.len + j;
      low[hh] = window_first(pos[hh], a.window);
      const __nv_bfloat16 *qr = (const __nv_bfloat16 *)a.q + ((long long)seg.b * a.c + j) * a.q_stride + h * HD + t4 * 2;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[ks][hh] = *reinterpret_cast<const uint32_t *>(qr + ks * 16);
        qf[ks][hh + 2] = *reinterpret_cast<const uint32_t *>(qr + ks * 16 + 8);
      }
    }
    const int p_first = seg.len + q0 / group, p_last = seg.len + q_last / group;
    const int low_first = window_first(p_first, a.window), low_last = window_first(p_last, a.window);
    float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f}, o[NB][4];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[n][x] = 0.f;

    for (; i < done + seg_n; i += W) {
      asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
      __syncwarp();                                      // everybody's copies are here, and the stage before is free
      request(stage == 0 ? S - 1 : stage - 1);
      const int key0 = tile_key(seg.k, seg.t + i - done, kKeys);
      const uint32_t kb = ring + stage * C::kTile, vb = kb + C::kHalf;
      const unsigned int bad = bad_keys[warp][stage];
      // ---- S = Q.K^T: 16 queries x 32 keys
      float s[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[n][x] = 0.f;
#pragma unroll
      for (int k2 = 0; k2 < KS / 2; ++k2) {
        uint32_t kf[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) ldsm4(kb + poff<HD>(n * 8 + (lane & 7), k2 * 4 + (lane >> 3)), kf[n]);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma16816(s[n], qf[2 * k2], kf[n][0], kf[n][1]);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma16816(s[n], qf[2 * k2 + 1], kf[n][2], kf[n][3]);
      }
      // ---- what the rows do not see, and keys without a page
      const bool masked = key0 + kKeys - 1 > p_first || (key0 < low_last && key0 + kKeys > a.n_sink);
      if (masked || bad) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int kk = n * 8 + t4 * 2 + (x & 1), t = key0 + kk;
            if (bad >> kk & 1u) s[n][x] = __int_as_float(0x7fffffff);
            if (t > pos[x >> 1] || (t < low[x >> 1] && t >= a.n_sink)) s[n][x] = -INFINITY;
          }
      }
      // ---- running maximum
      float mx[2] = {m_run[0], m_run[1]}, corr[2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        mx[0] = fmaxf(mx[0], fmaxf(s[n][0], s[n][1]));
        mx[1] = fmaxf(mx[1], fmaxf(s[n][2], s[n][3]));
      }
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        mx[hh] = fmaxf(mx[hh], __shfl_xor_sync(0xffffffffu, mx[hh], 1));
        mx[hh] = fmaxf(mx[hh], __shfl_xor_sync(0xffffffffu, mx[hh], 2));
        corr[hh] = mx[hh] == m_run[hh] ? 1.f : ex2((m_run[hh] - mx[hh]) * sl2);           // first tile: 2^-inf = 0
        m_run[hh] = mx[hh];
        l_run[hh] *= corr[hh];
      }
      // ---- probabilities
      const float mb[2] = {mx[0] == -INFINITY ? 0.f : mx[0] * sl2, mx[1] == -INFINITY ? 0.f : mx[1] * sl2};
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int x = 0; x < 4; ++x) s[n][x] = ex2(fmaf(s[n][x], sl2, -mb[x >> 1]));
        l_run[0] += s[n][0] + s[n][1];
        l_run[1] += s[n][2] + s[n][3];
      }
      // ---- values that are not finite, in a tile that some rows see more of than others: a probability of zero would
      // still carry them to the rows that do not see them.  Those keys are added row by row and taken out of the tile.
      if (masked && p_first != p_last) {
        unsigned int odd = 0;
        for (int e = lane; e < kKeys * PER; e += 32) {
          const int r = e / PER;
          const uint4 x = *reinterpret_cast<const uint4 *>(ring_g + (vb - ring) + poff<HD>(r, e % PER));
          const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if ((y[c] & 0x7f80u) == 0x7f80u || (y[c] & 0x7f800000u) == 0x7f800000u) odd |= 1u << r;
        }
        odd = __reduce_or_sync(0xffffffffu, odd);
        if (odd) {
#pragma unroll
          for (int n = 0; n < NB; ++n) { o[n][0] *= corr[0]; o[n][1] *= corr[0]; o[n][2] *= corr[1]; o[n][3] *= corr[1]; }
          corr[0] = corr[1] = 1.f;
          for (unsigned int left = odd; left; left &= left - 1) {
            const int kk = __ffs(left) - 1, t = key0 + kk;
            float p[2] = {0.f, 0.f};
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int x = 0; x < 4; ++x)
                if (n == kk >> 3 && (x & 1) == (kk & 1)) p[x >> 1] = s[n][x];
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
              p[hh] = __shfl_sync(0xffffffffu, p[hh], (lane & ~3) | ((kk & 7) >> 1));
              if (!sees(pos[hh], t, a.window, a.n_sink)) continue;
#pragma unroll
              for (int n = 0; n < NB; ++n) {
                const uint32_t y = *reinterpret_cast<const uint32_t *>(ring_g + (vb - ring) + poff<HD>(kk, n) + t4 * 4);
                o[n][2 * hh] = fmaf(p[hh], low_half(y), o[n][2 * hh]);
                o[n][2 * hh + 1] = fmaf(p[hh], high_half(y), o[n][2 * hh + 1]);
              }
            }
          }
          __syncwarp();
          for (int e = lane; e < kKeys * PER; e += 32)
            if (odd >> (e / PER) & 1u) *reinterpret_cast<uint4 *>(ring_g + (vb - ring) + poff<HD>(e / PER, e % PER)) = make_uint4(0, 0, 0, 0);
          __syncwarp();
        }
      }
      // ---- O = corr O + P.V, the score registers as the A operand
      uint32_t pf[NT / 2][3][4];
#pragma unroll
      for (int kk = 0; kk < NT / 2; ++kk)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          float p0 = s[2 * kk + (x >> 1)][(x & 1) * 2], p1 = s[2 * kk + (x >> 1)][(x & 1) * 2 + 1];
#pragma unroll
          for (int part = 0; part < 3; ++part) {
            pf[kk][part][x] = pack2(p0, p1);
            p0 -= low_half(pf[kk][part][x]);
            p1 -= high_half(pf[kk][part][x]);
          }
        }
#pragma unroll
      for (int n4 = 0; n4 < HD / 32; ++n4) {
        float y[4][4];
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x) y[n][x] = 0.f;
#pragma unroll
        for (int kk = 0; kk < NT / 2; ++kk) {
          uint32_t vf[2][4];
          ldsm4t(vb + poff<HD>(kk * 16 + (lane & 15), n4 * 4 + (lane >> 4)), vf[0]);
          ldsm4t(vb + poff<HD>(kk * 16 + (lane & 15), n4 * 4 + 2 + (lane >> 4)), vf[1]);
#pragma unroll
          for (int part = 2; part >= 0; --part)
#pragma unroll
            for (int n = 0; n < 4; ++n) mma16816(y[n], pf[kk][part], vf[n >> 1][(n & 1) * 2], vf[n >> 1][(n & 1) * 2 + 1]);
        }
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[4 * n4 + n][x] = fmaf(o[4 * n4 + n][x], corr[x >> 1], y[n][x]);
      }
      stage = stage + 1 == S ? 0 : stage + 1;
    }

    // ---- the warps' results: every warp adds up OWN column blocks
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      l_run[hh] += __shfl_xor_sync(0xffffffffu, l_run[hh], 1);
      l_run[hh] += __shfl_xor_sync(0xffffffffu, l_run[hh], 2);
    }
    if (t4 == 0) { ml[warp][g4] = make_float2(m_run[0], l_run[0]); ml[warp][g4 + 8] = make_float2(m_run[1], l_run[1]); }
#pragma unroll
    for (int w = 0; w < W; ++w)
      if (w != warp) {
#pragma unroll
        for (int n = 0; n < OWN; ++n)
          exchange[((w * (W - 1) + (warp < w ? warp : warp - 1)) * OWN + n) * 32 + lane] =
              make_float4(o[w * OWN + n][0], o[w * OWN + n][1], o[w * OWN + n][2], o[w * OWN + n][3]);
      }
    __syncthreads();
    float M[2], den[2], mine[2];
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      float2 v[W];
      M[hh] = -INFINITY;
#pragma unroll
      for (int w = 0; w < W; ++w) { v[w] = ml[w][g4 + 8 * hh]; M[hh] = fmaxf(M[hh], v[w].x); }
      den[hh] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) den[hh] = fmaf(v[w].y, v[w].x == -INFINITY && v[w].y == 0.f ? 0.f : ex2((v[w].x - M[hh]) * sl2), den[hh]);
      mine[hh] = m_run[hh] == -INFINITY && l_run[hh] == 0.f ? 0.f : ex2((m_run[hh] - M[hh]) * sl2);
    }
    float sum[OWN][4];
#pragma unroll
    for (int w = 0; w < W; ++w)
      if (w == warp) {
#pragma unroll
        for (int n = 0; n < OWN; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x) sum[n][x] = mine[x >> 1] * o[w * OWN + n][x];
      }
#pragma unroll
    for (int k = 0; k < W - 1; ++k) {
      const int w = k < warp ? k : k + 1;
      float f[2];
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const float2 v = ml[w][g4 + 8 * hh];
        f[hh] = v.x == -INFINITY && v.y == 0.f ? 0.f : ex2((v.x - M[hh]) * sl2);
      }
#pragma unroll
      for (int n = 0; n < OWN; ++n) {
        const float4 x = exchange[((warp * (W - 1) + k) * OWN + n) * 32 + lane];
        sum[n][0] = fmaf(f[0], x.x, sum[n][0]);
        sum[n][1] = fmaf(f[0], x.y, sum[n][1]);
        sum[n][2] = fmaf(f[1], x.z, sum[n][2]);
        sum[n][3] = fmaf(f[1], x.w, sum[n][3]);
      }
    }
    const bool whole = seg_n == seg.k.n;
    float *part = a.parts + ((long long)blockIdx.x * 2 + (done > 0)) * (16 * (HD + 2));
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int q = q0 + g4 + hh * 8;
      if (q >= nq) continue;
      const int j = q / group, h = kvh * group + q - j * group;
      const float f = whole ? result_scale(a, pos[hh], den[hh]) : 1.f;
      float *to = whole ? a.out + (((long long)seg.b * a.c + j) * a.hq + h) * HD : part + (g4 + hh * 8) * HD;
#pragma unroll
      for (int n = 0; n < OWN; ++n)
        *reinterpret_cast<float2 *>(to + (warp * OWN + n) * 8 + t4 * 2) = make_float2(sum[n][2 * hh] * f, sum[n][2 * hh + 1] * f);
      if (!whole && warp == 0 && t4 == 0) *reinterpret_cast<float2 *>(part + 16 * HD + (g4 + hh * 8) * 2) = make_float2(M[hh], den[hh]);
    }
    done += seg_n;
    if (done == n_mine) break;
    move_on(a, seg, seg_n);
    __syncthreads();                                     // the exchange buffers are free again
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

// ------------------------------------------------------------------------------------ joining the parts of a unit
// One block per unit: with items = queries x hd / 4 pieces of four columns, threads are groups that take turns at the parts.
constexpr int kCombine = 256;

template <int HD>
__global__ void __launch_bounds__(kCombine) paged_combine_kernel(const __grid_constant__ PagedAttnArgs a, int workers) {
  __shared__ long long counts[2];
  __shared__ float4 acc_s[kCombine];
  __shared__ float2 ml_s[kCombine];
  const int b = blockIdx.x / a.units, u = blockIdx.x - b * a.units, tid = threadIdx.x;
  int len;
  const KeyTiles k = seq_tiles(a, b, len);
  if (tid < 32) {
    long long total, before;
    count_tiles(a, b, total, before);
    if (tid == 0) { counts[0] = total; counts[1] = before; }
  }
  __syncthreads();
  const int group = a.hq / a.pool.n_kv_heads, nq = group * a.c, nqg = a.units / a.pool.n_kv_heads;
  const int kvh = u / nqg, q0 = (u - kvh * nqg) * 16, n_rows = min(16, nq - q0), items = n_rows * (HD / 4);
  const long long chunk = chunk_of(counts[0], workers), begin = counts[1] + (long long)u * k.n;
  UnitParts w = {0, -1};
  if (k.n > 0) {
    w = unit_parts(begin, k.n, chunk);
    if (w.first == w.last) return;                       // written by its one CTA
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
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
            const float *part = a.parts + ((long long)at * 2 + part_place(begin, at, chunk)) * (16 * (HD + 2));
            v[i] = __ldcg(reinterpret_cast<const float2 *>(part + 16 * HD + row * 2));
            x[i] = __ldcg(reinterpret_cast<const float4 *>(part + row * HD + c4 * 4));
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
          const float s = v[i].x == -INFINITY && v[i].y == 0.f ? 0.f : ex2((v[i].x - top) * sl2);
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
        float f = m == -INFINITY && den == 0.f ? 0.f : ex2((m - top) * sl2);
        den *= f; acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
        for (int i = 1; i < groups; ++i) {
          const float2 v = ml_s[tid + i * items];
          const float4 x = acc_s[tid + i * items];
          f = v.x == -INFINITY && v.y == 0.f ? 0.f : ex2((v.x - top) * sl2);
          den = fmaf(v.y, f, den);
          acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
        }
      }
    }
    if (e < items && g == 0) {
      const int q = q0 + row, j = q / group, h = kvh * group + q - j * group;
      const float f = len < 0 ? 0.f : result_scale(a, len + j, den);
      *reinterpret_cast<float4 *>(a.out + (((long long)b * a.c + j) * a.hq + h) * HD + c4 * 4) = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
    }
  }
}

// ------------------------------------------------------------------------------------ fp32: a block per row and query head
// The warps take turns at the keys, a lane holds HD / 32 elements.
template <int HD>
__global__ void __launch_bounds__(128) paged_fma_kernel(const __grid_constant__ PagedAttnArgs a) {
  constexpr int E = HD / 32;
  const int r = blockIdx.x, h = blockIdx.y, b = r / a.c, kvh = h / (a.hq / a.pool.n_kv_heads);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int len = clamp_len(a.kv_len[b], a.cap), p = len + (r - b * a.c);
  __shared__ float part[4][HD + 2];
  float q[E], o[E], m = -INFINITY, l = 0.f;
  const float *qr = (const float *)a.q + r * a.q_stride + h * HD + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) { q[e] = qr[e] * rsqrtf((float)HD); o[e] = 0.f; }
  const int32_t *row = a.table + (long long)b * a.width;
  const int first = len < 0 ? 0 : window_first(p, a.window), sinks = len < 0 ? 0 : min(a.n_sink, first);
  const int n = len < 0 ? 0 : sinks + p + 1 - first;
  for (int i = warp; i < n; i += 4) {
    const int t = i < sinks ? i : first + i - sinks;
    const int page = page_of(row, a.width, t, a.pool.page_size, a.pool.n_pages);
    const long long at = (long long)page * a.pool.page_stride + kvh * a.pool.head_stride + (t % a.pool.page_size) * a.pool.slot_stride + lane * E;
    float s = 0.f, v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      s = fmaf(q[e], page < 0 ? NAN : ((const float *)a.pool.k)[at + e], s);
      v[e] = page < 0 ? NAN : ((const float *)a.pool.v)[at + e];
    }
#pragma unroll
    for (int k = 16; k; k >>= 1) s += __shfl_xor_sync(0xffffffffu, s, k);
    const float mn = fmaxf(m, s), f = m == -INFINITY ? 0.f : expf(m - mn), w = expf(s - mn);
    l = l * f + w;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + w * v[e];
    m = mn;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) part[warp][lane * E + e] = o[e];
  if (lane == 0) { part[warp][HD] = m; part[warp][HD + 1] = l; }
  __syncthreads();
  for (int e = threadIdx.x; e < HD; e += 128) {
    float M = -INFINITY, den = 0.f, sum = 0.f;
    for (int w = 0; w < 4; ++w) M = fmaxf(M, part[w][HD]);
    for (int w = 0; w < 4; ++w) {
      const float f = part[w][HD] == -INFINITY && part[w][HD + 1] == 0.f ? 0.f : expf(part[w][HD] - M);
      den += f * part[w][HD + 1];
      sum += f * part[w][e];
    }
    a.out[((long long)r * a.hq + h) * HD + e] = den == 0.f ? 0.f : sum / den;
  }
}

// ------------------------------------------------------------------------------------ host side
template <int HD>
cudaError_t launch_mma(const PagedAttnArgs &a, int workers, cudaStream_t st) {
  using C = PagedCfg<HD>;
  static bool attr_done[kMaxDevices] = {false};
  const int dev = current_device_slot();
  if (!attr_done[dev]) {
    if (cudaError_t e = cudaFuncSetAttribute(paged_mma_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmem)) return e;
    attr_done[dev] = true;
  }
  paged_mma_kernel<HD><<<workers, C::W * 32, C::kSmem, st>>>(a);
  if (cudaError_t e = cudaGetLastError()) return e;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3((unsigned)(a.batch * a.units)); cfg.blockDim = dim3(kCombine); cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, paged_combine_kernel<HD>, a, workers);
}

template <int HD>
cudaError_t launch_fma(const PagedAttnArgs &a, cudaStream_t st) {
  paged_fma_kernel<HD><<<dim3(a.batch * a.c, a.hq), 128, 0, st>>>(a);
  return cudaGetLastError();
}

constexpr int kWorkers = 148;

}  // namespace

size_t paged_attn_scratch(int hd, int dtype) { return dtype == FC_F32 ? 256 : (size_t)kWorkers * 2 * 16 * (hd + 2) * sizeof(float); }

cudaError_t launch_paged_attn(PagedAttnArgs a, int dtype, int hd, cudaStream_t st) {
  const int group = a.hq / a.pool.n_kv_heads;
  a.units = a.pool.n_kv_heads * ((group * a.c + 15) / 16);
  if (dtype == FC_F32) return hd == 128 ? launch_fma<128>(a, st) : hd == 64 ? launch_fma<64>(a, st) : launch_fma<32>(a, st);
  return hd == 128 ? launch_mma<128>(a, kWorkers, st) : hd == 64 ? launch_mma<64>(a, kWorkers, st) : launch_mma<32>(a, kWorkers, st);
}

}  // namespace fc
