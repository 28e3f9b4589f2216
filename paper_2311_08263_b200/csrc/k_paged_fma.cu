// Window attention over pages in fp32: the line, the clusters and the rings of k_paged_attn.cu with FMA instead of MMA.
//
// A tile is 1024 elements of keys and as many of values (8, 16 or 32 keys at hd 128, 64, 32).  Scores: a lane takes one key and 32 elements of it, for
// all queries of the unit, whose rows lie in shared memory.  Output: a lane takes hd / 32 elements of all queries; probabilities come from shared
// memory, four queries at a time.  Up to eight queries a unit the K/V stream is the bound; more queries are more units, which find it in L2.
// Measured: 16 x 32 kv heads x 1 query over 2048 keys of hd 128 163 us (6.6 TB/s); 4 kv heads x 8 queries over 32000 keys of hd 64 30 us (2.2 TB/s, FMA and shared memory);
// 16 x 4 x 128 queries over 641 keys of hd 64 104 us.
#include "fc_paged.cuh"

namespace fc {

namespace {

constexpr int kWarps = kPagedWarps, kThreads = kWarps * 32;

template <int HD, int QB>
struct FmaCfg {
  static constexpr int KEYS = 1024 / HD, kRow = HD * 4, S = 3;
  static constexpr uint32_t kHalf = 4096, kTile = 2 * kHalf;
  static constexpr uint32_t kRing = kWarps * S * kTile;
  static constexpr uint32_t kQ = QB * HD * 4;                       // the unit's queries
  static constexpr uint32_t kP = kWarps * KEYS * QB * 4;            // probabilities, per warp [key][query]
  static constexpr int XQ = QB < 4 ? QB : 4;                        // queries that are exchanged at a time
  static constexpr uint32_t kExchange = kWarps * XQ * HD * 4;
  static constexpr size_t kSmem = 128 + kRing + kP + (kQ + kExchange > kWarps * kQ ? kQ + kExchange : kWarps * kQ);
};

template <int HD, int QB, bool LINE>
__global__ void __launch_bounds__(kThreads, 1) paged_fma_kernel(const __grid_constant__ PagedAttnArgs a) {
  using C = FmaCfg<HD, QB>;
  constexpr int W = kWarps, S = C::S, KEYS = C::KEYS, E = HD / 32;
  if (LINE) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ unsigned char smem_raw[];
  __shared__ float2 ml[W][QB], ml_cta[QB];               // (max, sum)
  __shared__ unsigned int bad_keys[W][S];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t base = (smem_u32(smem_raw) + 127u) & ~127u;
  unsigned char *base_g = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t ring = base + (uint32_t)warp * (S * C::kTile);
  float *ps = reinterpret_cast<float *>(base_g + C::kRing) + warp * KEYS * QB;
  // the unit's queries, and room for the exchange; a warp on its own has its queries where the others would exchange
  float *qs = reinterpret_cast<float *>(base_g + C::kRing + C::kP) + (LINE ? warp * QB * HD : 0);
  float *exchange = reinterpret_cast<float *>(base_g + C::kRing + C::kP + C::kQ);

  const int group = a.group, nq = a.nq;
  const float sl2 = rsqrtf((float)HD) * 1.4426950408889634f;
  Place seg;
  int n_mine;
  const int worker = warp * kSms + (int)blockIdx.x;      // on the line: consecutive pieces on different SMs
  if (!my_piece<KEYS, LINE>(a, worker, W * kSms, seg, n_mine)) return;
  constexpr int STEP = LINE ? 1 : W;
  TileStream<KEYS, C::kRow, S, QB, LINE, W> stream(a, seg, LINE ? 0 : warp, n_mine, ring, bad_keys[warp]);
#pragma unroll 1
  for (int s = 0; s < S - 1; ++s) stream.request(s);

  const int key = lane % KEYS, share = lane / KEYS;      // a lane's key, and which 32 elements of it
  int stage = 0, i = LINE ? 0 : warp, done = 0;
  while (true) {
    // ---- a segment: tiles done .. done + seg_n of the piece, tiles seg.t .. of the unit
    const int seg_n = min(n_mine - done, seg.k.n - seg.t);
    const int q0 = seg.qg * QB, q_last = min(nq - 1, q0 + QB - 1);
    // on the line the warps have places of their own for the queries
    if (LINE) __syncwarp();
    for (int e = LINE ? lane : tid; e < QB * (HD / 4); e += LINE ? 32 : kThreads) {
      const int n = e / (HD / 4), c4 = e - n * (HD / 4), q = min(q0 + n, nq - 1), j = quotient16(q, a.group_inv), h = seg.kvh * group + q - j * group;
      reinterpret_cast<float4 *>(qs)[e] = *reinterpret_cast<const float4 *>((const float *)a.q + ((long long)seg.b * a.c + j) * a.q_stride + h * HD + c4 * 4);
    }
    if (LINE) __syncwarp();
    else __syncthreads();
    int pos[QB];
    float m[QB], l[QB], o[QB][E];
#pragma unroll
    for (int n = 0; n < QB; ++n) {
      pos[n] = seg.len + quotient16(min(q0 + n, nq - 1), a.group_inv);
      m[n] = -INFINITY;
      l[n] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[n][e] = 0.f;
    }
    const int p_first = seg.len + quotient16(q0, a.group_inv), p_last = seg.len + quotient16(q_last, a.group_inv), low_last = window_first(p_last, a.window);

    for (; i < done + seg_n; i += STEP) {
      asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
      __syncwarp();                                      // everybody's copies are here, and the stage before is free
      stream.request(stage == 0 ? S - 1 : stage - 1);
      const int key0 = tile_key(seg.k, seg.t + i - done, KEYS);
      const unsigned char *kt = base_g + (ring + stage * C::kTile - base), *vt = kt + C::kHalf;
      const unsigned int bad = bad_keys[warp][stage];
      // ---- scores
      float s[QB];
#pragma unroll
      for (int n = 0; n < QB; ++n) s[n] = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float4 x = *reinterpret_cast<const float4 *>(kt + poff<KEYS, C::kRow>(key, share * 8 + c));
#pragma unroll
        for (int n = 0; n < QB; ++n) {
          const float4 y = *reinterpret_cast<const float4 *>(qs + n * HD + share * 32 + c * 4);
          s[n] = fmaf(x.x, y.x, s[n]); s[n] = fmaf(x.y, y.y, s[n]); s[n] = fmaf(x.z, y.z, s[n]); s[n] = fmaf(x.w, y.w, s[n]);
        }
      }
      const bool masked = key0 + KEYS - 1 > p_first || (key0 < low_last && key0 + KEYS > a.n_sink);
      float corr[QB];
#pragma unroll
      for (int n = 0; n < QB; ++n) {
#pragma unroll
        for (int d = KEYS; d < 32; d <<= 1) s[n] += __shfl_xor_sync(0xffffffffu, s[n], d);
        if (bad >> lane & 1u) s[n] = quiet_nan();
        if (masked && !sees(pos[n], key0 + key, a.window, a.n_sink)) s[n] = -INFINITY;
        float mx = fmaxf(m[n], s[n]);
#pragma unroll
        for (int d = 1; d < KEYS; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        corr[n] = mx == m[n] ? 1.f : ex2((m[n] - mx) * sl2);
        m[n] = mx;
        s[n] = ex2(fmaf(s[n], sl2, mx == -INFINITY ? 0.f : -mx * sl2));
        l[n] = fmaf(l[n], corr[n], s[n]);                // of this lane's key; added up at the end
#pragma unroll
        for (int e = 0; e < E; ++e) o[n][e] *= corr[n];
      }
      if (share == 0) {
#pragma unroll
        for (int n = 0; n < QB; n += QB < 4 ? 1 : 4) {
          if (QB < 4) ps[key * QB + n] = s[n];
          else *reinterpret_cast<float4 *>(ps + key * QB + n) = make_float4(s[n], s[(n + 1) % QB], s[(n + 2) % QB], s[(n + 3) % QB]);
        }
      }
      __syncwarp();
      // ---- output.  Where rows see different keys of the tile and some value is not finite, what a row does not see is not even multiplied.
      bool apart = false;
      if (masked && p_first != p_last) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float4 x = *reinterpret_cast<const float4 *>(vt + (e * 32 + lane) * 16);
          apart |= !(fabsf(x.x) < INFINITY && fabsf(x.y) < INFINITY && fabsf(x.z) < INFINITY && fabsf(x.w) < INFINITY);
        }
        apart = __any_sync(0xffffffffu, apart);
      }
      auto value = [&](int k, float (&v)[E]) {
        if (E == 4) {
          const float4 x = *reinterpret_cast<const float4 *>(vt + poff<KEYS, C::kRow>(k, lane));
          v[0] = x.x; v[E > 1 ? 1 : 0] = x.y; v[E > 2 ? 2 : 0] = x.z; v[E > 3 ? 3 : 0] = x.w;
        } else if (E == 2) {
          const float2 x = *reinterpret_cast<const float2 *>(vt + poff<KEYS, C::kRow>(k, lane >> 1) + (lane & 1) * 8);
          v[0] = x.x; v[E > 1 ? 1 : 0] = x.y;
        } else {
          v[0] = *reinterpret_cast<const float *>(vt + poff<KEYS, C::kRow>(k, lane >> 2) + (lane & 3) * 4);
        }
      };
      if (apart) {
        for (int k = 0; k < KEYS; ++k) {
          float v[E];
          value(k, v);
#pragma unroll
          for (int n = 0; n < QB; ++n)
            if (sees(pos[n], key0 + k, a.window, a.n_sink)) {
#pragma unroll
              for (int e = 0; e < E; ++e) o[n][e] = fmaf(ps[k * QB + n], v[e], o[n][e]);
            }
        }
      } else {
#pragma unroll 8
        for (int k = 0; k < KEYS; ++k) {
          float v[E], p[QB];
          value(k, v);
          if (QB == 8) {
            const float4 x = *reinterpret_cast<const float4 *>(ps + k * QB), y = *reinterpret_cast<const float4 *>(ps + k * QB + 4);
            p[0] = x.x; p[1 % QB] = x.y; p[2 % QB] = x.z; p[3 % QB] = x.w; p[4 % QB] = y.x; p[5 % QB] = y.y; p[6 % QB] = y.z; p[7 % QB] = y.w;
          } else {
            p[0] = ps[k];
          }
#pragma unroll
          for (int n = 0; n < QB; ++n)
#pragma unroll
            for (int e = 0; e < E; ++e) o[n][e] = fmaf(p[n], v[e], o[n][e]);
        }
      }
      __syncwarp();                                      // the probabilities' place is written again
      stage = stage + 1 == S ? 0 : stage + 1;
    }

    // ---- the warps' results, some queries at a time
#pragma unroll
    for (int n = 0; n < QB; ++n) {
#pragma unroll
      for (int d = 1; d < KEYS; d <<= 1) l[n] += __shfl_xor_sync(0xffffffffu, l[n], d);
      if (!LINE && lane == 0) ml[warp][n] = make_float2(m[n], l[n]);
    }
    if (!LINE) asm volatile("cp.async.wait_all;" ::: "memory");
    const bool whole = LINE ? seg_n == seg.k.n : gridDim.x == 1;
    if (LINE) {
      // ---- all of it is this warp's
      float *part = a.parts + ((long long)worker * 2 + (done > 0)) * part_floats(QB, HD);
#pragma unroll
      for (int n = 0; n < QB; ++n) {
        const int q = q0 + n;
        if (q >= nq) continue;
        const int j = quotient16(q, a.group_inv), h = seg.kvh * group + q - j * group;
        const float f = whole ? result_scale(a, pos[n], l[n]) : 1.f;
        float *to = whole ? a.out + (((long long)seg.b * a.c + j) * a.hq + h) * HD : part + n * HD;
#pragma unroll
        for (int e = 0; e < E; ++e) to[lane * E + e] = o[n][e] * f;
        if (!whole && lane == 0) *reinterpret_cast<float2 *>(part + QB * HD + n * 2) = make_float2(m[n], l[n]);
      }
      done += seg_n;
      if (done == n_mine) break;
      move_on<KEYS>(a, seg, seg_n);
      continue;
    }
    // sums that are not the whole unit's: this CTA's shared memory (the ring, drained)
    float *part = reinterpret_cast<float *>(base_g);
#pragma unroll
    for (int n0 = 0; n0 < QB; n0 += C::XQ) {
      if (n0) __syncthreads();
#pragma unroll
      for (int n = 0; n < C::XQ; ++n)
#pragma unroll
        for (int e = 0; e < E; ++e) exchange[(warp * C::XQ + n) * HD + lane * E + e] = o[n0 + n][e];
      __syncthreads();
      for (int e = tid; e < C::XQ * (HD / 4); e += kThreads) {
        const int x = e / (HD / 4), c4 = e - x * (HD / 4), n = n0 + x, q = q0 + n, j = quotient16(q, a.group_inv), h = seg.kvh * group + q - j * group;
        if (q >= nq) continue;
        float M = -INFINITY, den = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < W; ++w) M = fmaxf(M, ml[w][n].x);
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const float f = part_weight(ml[w][n], M, sl2);
          const float4 y = *reinterpret_cast<const float4 *>(exchange + (w * C::XQ + x) * HD + c4 * 4);
          den = fmaf(ml[w][n].y, f, den);
          acc.x = fmaf(f, y.x, acc.x); acc.y = fmaf(f, y.y, acc.y); acc.z = fmaf(f, y.z, acc.z); acc.w = fmaf(f, y.w, acc.w);
        }
        const float f = !whole ? 1.f : seg.len < 0 ? 0.f : result_scale(a, seg.len + j, den);
        float *to = whole ? a.out + (((long long)seg.b * a.c + j) * a.hq + h) * HD : part + n * HD;
        *reinterpret_cast<float4 *>(to + c4 * 4) = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
        if (!whole && c4 == 0) ml_cta[n] = make_float2(M, den);
      }
    }
    break;
  }
  if (LINE) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    return;
  }
  if (gridDim.x == 1) return;
  const int q0 = seg.qg * QB;
  join_cluster<HD>(a, seg, q0, min(QB, nq - q0), base, smem_u32(ml_cta), kThreads);
}

template <int HD, int QB>
cudaError_t launch(const PagedAttnArgs &a, const PagedPlan &plan, cudaStream_t st) {
  using C = FmaCfg<HD, QB>;
  static bool done[2][kMaxDevices] = {};
  return launch_units<HD, QB, C::KEYS>(a, plan, paged_fma_kernel<HD, QB, true>, paged_fma_kernel<HD, QB, false>, C::kSmem, done, st);
}
template <int HD>
cudaError_t launch_hd(const PagedAttnArgs &a, const PagedPlan &plan, cudaStream_t st) {
  return plan.queries == 1 ? launch<HD, 1>(a, plan, st) : launch<HD, 8>(a, plan, st);
}

}  // namespace

cudaError_t launch_paged_fma(const PagedAttnArgs &a, const PagedPlan &plan, int hd, cudaStream_t st) {
  return hd == 128 ? launch_hd<128>(a, plan, st) : hd == 64 ? launch_hd<64>(a, plan, st) : launch_hd<32>(a, plan, st);
}

}  // namespace fc
