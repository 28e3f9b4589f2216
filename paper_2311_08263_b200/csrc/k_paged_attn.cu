// Window attention over pages: out = softmax(q.k / sqrt(hd)) v over the keys that a row sees, keys and values behind a table of pages.
//
// paged_mma_kernel (bf16).  A unit is a kv head of a sequence and 8 or 16 queries (window rows x heads of the group); its keys come in tiles of
// 16.  The products are taken with the keys as rows, S^T = K.Q^T and O^T = V^T.P^T, so that the 16 rows of an MMA are keys and
// head elements, always full, and only its 8 columns are queries.  A warp loads its own tiles into its own ring (cp.async, 16 bytes a lane; the
// lanes look up the pages of the tile's keys, a tile ahead), so that it waits for nobody while it streams.  Scores, probabilities and the output
// stay in its registers.
//   Line: one CTA per SM, eight or twelve warps (more_warps_pay).  The tiles of all units stand in one line, sequence by sequence, cut into equal pieces, one per warp,
// whatever the lengths: the launch depends on none, a batch of ragged caches is as balanced as one long cache, and the rings run on from unit to
// unit.  A unit that several warps share goes to scratch as un-normalised sums, which paged_combine_kernel adds up in order.
//   (A piece per CTA, whose warps take turns at its tiles and exchange sums where a unit ends, leaves fewer parts but stalls at every end: 7B, 16 x 1 token over
// 2048 keys 88 us against 79, 40 x 8 rows over 10 keys 52 against 12; only one sequence over 32000 keys was better, 87.6 against 91.)
//   Cluster: for tables that hold little, a cluster per unit, whose warps take turns at the tiles.  They exchange their sums through shared memory, each
// adds up a part of the elements, and the CTAs join theirs through distributed shared memory: one launch, no scratch.
// Bound by HBM where there is much to read (7B, 16 x 1 token over 2048 keys: 78 us, 6.1 TB/s), by latency below some 50 MB.
//
// Probabilities enter the tensor cores as three bf16 parts (their sum has all 24 bits), a tile's product is added to the output in fp32: what is rounded
// is what is stored in the cache, nothing else.  (Two parts leave 1.5e-6, relative, of the result.)
// An infinite value that a row sees becomes NaN where it meets parts of zero or of the other sign, which only tiles that some row does not see whole
// rule out (their values that are not finite are added by FMA): no finite result either way, and more is not promised.
#include "fc_paged.cuh"

namespace fc {

namespace {

constexpr int kKeys = kMmaKeys;        // per tile

// W: warps of a CTA
template <int HD, int W>
struct PagedCfg {
  static constexpr int kThreads = W * 32;
  static constexpr int kRow = HD * 2;                              // bytes of a key
  static constexpr uint32_t kHalf = kKeys * kRow, kTile = 2 * kHalf;
  static constexpr int S = HD == 32 ? 6 : HD == 64 ? 48 / W : 24 / W;      // stages of a warp's ring: 192 KB in all, at hd 32 96 or (12 warps) 144
  static constexpr int DB = HD / 16;                               // blocks of 16 elements of the output
  static constexpr uint32_t kRing = W * S * kTile;
  // Of a cluster, a block of 8 queries at a time.  The line of eight warps asks for it too: SMs are then set to all the shared memory they can have, and the joining
  // kernel's blocks fit in beside (1 sequence x 4 kv heads over 32000 keys 14.5 us, 15.6 without); twelve warps are faster alone (8 x 40 x 16 queries over 1024 48.4, 50.6).
  static constexpr uint32_t kExchange = W > kPagedWarps ? 0 : DB * (W - 1) * 512;
  static constexpr size_t kSmem = 128 + kRing + kExchange;
};

// 8 x 8 transpose of 16-bit elements across a warp
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

// QN: blocks of 8 queries of a unit.  W: warps.  LINE: the line of tiles, else a cluster per unit (grid: CTAs of the cluster, units, sequences).
template <int HD, int QN, int W, bool LINE>
__global__ void __launch_bounds__(W * 32, 1) paged_mma_kernel(const __grid_constant__ PagedAttnArgs a) {
  using C = PagedCfg<HD, W>;
  constexpr int S = C::S, KS = HD / 16, DB = C::DB, Q = 8 * QN;
  constexpr int PER = HD / 8;                            // 16-byte pieces of a row
  constexpr int OWN = (DB + W - 1) / W;                  // blocks of elements that a warp adds up
  if (LINE) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ unsigned char smem_raw[];
  __shared__ float2 ml[W][Q];                            // (max, sum) per warp and query
  __shared__ unsigned int bad_keys[W][S];                // keys of a tile whose page is missing
  __shared__ float2 ml_cta[Q];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g4 = lane >> 2, t4 = lane & 3;
  const uint32_t base = (smem_u32(smem_raw) + 127u) & ~127u;
  unsigned char *base_g = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t ring = base + (uint32_t)warp * (S * C::kTile);
  float4 *exchange = reinterpret_cast<float4 *>(base_g + C::kRing);

  const int group = a.group, nq = a.nq;
  const float sl2 = rsqrtf((float)HD) * 1.4426950408889634f;
  Place seg;                                             // where the segment (a unit's tiles in this CTA's piece) begins
  int n_mine;
  const int worker = warp * kSms + (int)blockIdx.x;      // on the line: consecutive pieces on different SMs
  if (!my_piece<kKeys, LINE>(a, worker, W * kSms, seg, n_mine)) return;
  constexpr int STEP = LINE ? 1 : W;
  TileStream<kKeys, C::kRow, S, Q, LINE, W> stream(a, seg, LINE ? 0 : warp, n_mine, ring, bad_keys[warp]);
#pragma unroll 1
  for (int s = 0; s < S - 1; ++s) stream.request(s);

  int stage = 0;
  int i = LINE ? 0 : warp;                               // this warp's next tile in the piece
  int done = 0;                                          // tiles of the piece in front of the segment
  while (true) {
    // ---- a segment: tiles done .. done + seg_n of the piece, tiles seg.t .. of the unit
    const int seg_n = min(n_mine - done, seg.k.n - seg.t);
    const int q0 = seg.qg * Q, q_last = min(nq - 1, q0 + Q - 1);
    // a lane's queries as columns of the scores: 2 t4 and 2 t4 + 1 of each block; as columns of Q^T: g4
    int pos[QN][2], low[QN][2];
    uint32_t qf[QN][KS][2];
#pragma unroll
    for (int n = 0; n < QN; ++n) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        pos[n][x] = seg.len + quotient16(min(q0 + n * 8 + t4 * 2 + x, nq - 1), a.group_inv);
        low[n][x] = window_first(pos[n][x], a.window);
      }
      const int q = min(q0 + n * 8 + g4, nq - 1), j = quotient16(q, a.group_inv), h = seg.kvh * group + q - j * group;
      const __nv_bfloat16 *qr = (const __nv_bfloat16 *)a.q + ((long long)seg.b * a.c + j) * a.q_stride + h * HD + t4 * 2;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[n][ks][0] = *reinterpret_cast<const uint32_t *>(qr + ks * 16);
        qf[n][ks][1] = *reinterpret_cast<const uint32_t *>(qr + ks * 16 + 8);
      }
    }
    const int p_first = seg.len + quotient16(q0, a.group_inv), p_last = seg.len + quotient16(q_last, a.group_inv);
    const int low_last = window_first(p_last, a.window);
    float m_run[QN][2], l_run[QN][2], o[QN][DB][4];
#pragma unroll
    for (int n = 0; n < QN; ++n) {
      m_run[n][0] = m_run[n][1] = -INFINITY;
      l_run[n][0] = l_run[n][1] = 0.f;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[n][d][x] = 0.f;
    }

    for (; i < done + seg_n; i += STEP) {
      asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
      __syncwarp();                                      // everybody's copies are here, and the stage before is free
      stream.request(stage == 0 ? S - 1 : stage - 1);
      const int key0 = tile_key(seg.k, seg.t + i - done, kKeys);
      const uint32_t kb = ring + stage * C::kTile, vb = kb + C::kHalf;
      const unsigned int bad = bad_keys[warp][stage];
      // ---- S^T = K.Q^T: 16 keys x 8 QN queries; the k range in two halves (shorter chains of MMAs)
      float s[QN][4], s2[QN][4];
#pragma unroll
      for (int n = 0; n < QN; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[n][x] = s2[n][x] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ks += 2) {
        uint32_t k0[4], k1[4];
        ldsm4(kb + poff<kKeys, C::kRow>(lane & 15, ks * 2 + (lane >> 4)), k0);
        ldsm4(kb + poff<kKeys, C::kRow>(lane & 15, ks * 2 + 2 + (lane >> 4)), k1);
#pragma unroll
        for (int n = 0; n < QN; ++n) mma16816(s[n], k0, qf[n][ks][0], qf[n][ks][1]);
#pragma unroll
        for (int n = 0; n < QN; ++n) mma16816(s2[n], k1, qf[n][ks + 1][0], qf[n][ks + 1][1]);
      }
#pragma unroll
      for (int n = 0; n < QN; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[n][x] += s2[n][x];
      // ---- what the rows do not see, and keys without a page
      const bool masked = key0 + kKeys - 1 > p_first || (key0 < low_last && key0 + kKeys > a.n_sink);
      if (masked || bad) {
#pragma unroll
        for (int n = 0; n < QN; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int kk = g4 + (x >> 1) * 8, t = key0 + kk;
            if (bad >> kk & 1u) s[n][x] = quiet_nan();
            if (t > pos[n][x & 1] || (t < low[n][x & 1] && t >= a.n_sink)) s[n][x] = -INFINITY;
          }
      }
      // ---- running maximum of the lane's queries
      float corr[QN][2];
#pragma unroll
      for (int n = 0; n < QN; ++n)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float mx = fmaxf(m_run[n][x], fmaxf(s[n][x], s[n][x + 2]));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          corr[n][x] = mx == m_run[n][x] ? 1.f : ex2((m_run[n][x] - mx) * sl2);           // first tile: 2^-inf = 0
          m_run[n][x] = mx;
          const float mb = mx == -INFINITY ? 0.f : mx * sl2;
          s[n][x] = ex2(fmaf(s[n][x], sl2, -mb));
          s[n][x + 2] = ex2(fmaf(s[n][x + 2], sl2, -mb));
          l_run[n][x] = fmaf(l_run[n][x], corr[n][x], s[n][x] + s[n][x + 2]);
        }
      // ---- values that are not finite, in a tile that some rows see more of than others: a probability of zero would
      // still carry them to the rows that do not see them.  Those keys are added row by row and taken out of the tile.
      if (masked && p_first != p_last) {
        unsigned char *vg = base_g + (vb - base);
        unsigned int odd = 0;
        for (int e = lane; e < kKeys * PER; e += 32) {
          const uint4 x = *reinterpret_cast<const uint4 *>(vg + poff<kKeys, C::kRow>(e / PER, e % PER));
          const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int w = 0; w < 4; ++w)
            if ((y[w] & 0x7f80u) == 0x7f80u || (y[w] & 0x7f800000u) == 0x7f800000u) odd |= 1u << (e / PER);
        }
        odd = __reduce_or_sync(0xffffffffu, odd);
        if (odd) {
#pragma unroll
          for (int n = 0; n < QN; ++n)
#pragma unroll
            for (int x = 0; x < 2; ++x) {                // rows that see none of them are computed as ever
              bool hit = false;
              for (unsigned int left = odd; left; left &= left - 1) hit |= sees(pos[n][x], key0 + __ffs(left) - 1, a.window, a.n_sink);
              if (!hit) continue;
#pragma unroll
              for (int d = 0; d < DB; ++d) {
                o[n][d][x] *= corr[n][x];
                o[n][d][x + 2] *= corr[n][x];
              }
              corr[n][x] = 1.f;
            }
          for (unsigned int left = odd; left; left &= left - 1) {
            const int kk = __ffs(left) - 1;
#pragma unroll
            for (int n = 0; n < QN; ++n)
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                const float p = __shfl_sync(0xffffffffu, kk < 8 ? s[n][x] : s[n][x + 2], (kk & 7) * 4 + t4);
                if (!sees(pos[n][x], key0 + kk, a.window, a.n_sink)) continue;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                  for (int e = 0; e < 2; ++e) {
                    const __nv_bfloat16 y = *reinterpret_cast<const __nv_bfloat16 *>(vg + poff<kKeys, C::kRow>(kk, d * 2 + e) + g4 * 2);
                    o[n][d][2 * e + x] = fmaf(p, __bfloat162float(y), o[n][d][2 * e + x]);
                  }
              }
          }
          __syncwarp();
          for (int e = lane; e < kKeys * PER; e += 32)
            if (odd >> (e / PER) & 1u) *reinterpret_cast<uint4 *>(vg + poff<kKeys, C::kRow>(e / PER, e % PER)) = make_uint4(0, 0, 0, 0);
          __syncwarp();
        }
      }
      // ---- O^T = corr O^T + V^T.P^T; the scores' registers, transposed in 8 x 8 blocks, are the B operand
      uint32_t pf[QN][3][2];
#pragma unroll
      for (int n = 0; n < QN; ++n)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float p0 = s[n][2 * x], p1 = s[n][2 * x + 1];
#pragma unroll
          for (int part = 0; part < 3; ++part) {
            const uint32_t y = pack2(p0, p1);
            p0 -= low_half(y);
            p1 -= high_half(y);
            pf[n][part][x] = transpose8(y);
          }
        }
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        uint32_t vf[4];
        ldsm4t(vb + poff<kKeys, C::kRow>((lane & 7) + ((lane >> 4) << 3), d * 2 + ((lane >> 3) & 1)), vf);
        float y[QN][4];
#pragma unroll
        for (int n = 0; n < QN; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x) y[n][x] = 0.f;
#pragma unroll
        for (int part = 2; part >= 0; --part)
#pragma unroll
          for (int n = 0; n < QN; ++n) mma16816(y[n], vf, pf[n][part][0], pf[n][part][1]);
#pragma unroll
        for (int n = 0; n < QN; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[n][d][x] = fmaf(o[n][d][x], corr[n][x & 1], y[n][x]);
      }
      stage = stage + 1 == S ? 0 : stage + 1;
    }

    // ---- the warps' results, a block of queries at a time: warp w adds up element blocks w, w + W ..
#pragma unroll
    for (int n = 0; n < QN; ++n)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        l_run[n][x] += __shfl_xor_sync(0xffffffffu, l_run[n][x], 4);
        l_run[n][x] += __shfl_xor_sync(0xffffffffu, l_run[n][x], 8);
        l_run[n][x] += __shfl_xor_sync(0xffffffffu, l_run[n][x], 16);
        if (!LINE && g4 == 0) ml[warp][n * 8 + t4 * 2 + x] = make_float2(m_run[n][x], l_run[n][x]);
      }
    const bool whole = LINE ? seg_n == seg.k.n : gridDim.x == 1;
    if (LINE) {
      // ---- all of it is this warp's
      float *part = a.parts + ((long long)worker * 2 + (done > 0)) * part_floats(Q, HD);
#pragma unroll
      for (int n = 0; n < QN; ++n)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int q = q0 + n * 8 + t4 * 2 + x;
          if (q >= nq) continue;
          const int j = quotient16(q, a.group_inv), h = seg.kvh * group + q - j * group;
          const float f = whole ? result_scale(a, pos[n][x], l_run[n][x]) : 1.f;
          float *to = whole ? a.out + (((long long)seg.b * a.c + j) * a.hq + h) * HD : part + (q - q0) * HD;
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            to[d * 16 + g4] = o[n][d][x] * f;
            to[d * 16 + g4 + 8] = o[n][d][x + 2] * f;
          }
          if (!whole && g4 == 0) *reinterpret_cast<float2 *>(part + Q * HD + (q - q0) * 2) = make_float2(m_run[n][x], l_run[n][x]);
        }
      done += seg_n;
      if (done == n_mine) break;
      move_on<kKeys>(a, seg, seg_n);
      continue;
    }
    // sums that are not the whole unit's: this CTA's shared memory (the ring, drained)
    float *part = reinterpret_cast<float *>(base_g);
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int n = 0; n < QN; ++n) {
      if (n) __syncthreads();
#pragma unroll
      for (int d = 0; d < DB; ++d)
        if (d % W != warp) exchange[(d * (W - 1) + (warp < d % W ? warp : warp - 1)) * 32 + lane] = make_float4(o[n][d][0], o[n][d][1], o[n][d][2], o[n][d][3]);
      __syncthreads();
      float M[2], den[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        M[x] = -INFINITY;
        den[x] = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) M[x] = fmaxf(M[x], ml[w][n * 8 + t4 * 2 + x].x);
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const float2 v = ml[w][n * 8 + t4 * 2 + x];
          den[x] = fmaf(v.y, part_weight(v, M[x], sl2), den[x]);
        }
      }
#pragma unroll
      for (int k = 0; k < OWN; ++k) {
        const int d = k * W + warp;
        if (d >= DB) break;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < W; ++w) {
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
          if (w != warp) x = exchange[(d * (W - 1) + (w < warp ? w : w - 1)) * 32 + lane];
          else {
#pragma unroll
            for (int e = 0; e < DB; ++e)
              if (e == d) x = make_float4(o[n][e][0], o[n][e][1], o[n][e][2], o[n][e][3]);
          }
          const float f0 = part_weight(ml[w][n * 8 + t4 * 2], M[0], sl2), f1 = part_weight(ml[w][n * 8 + t4 * 2 + 1], M[1], sl2);
          sum[0] = fmaf(f0, x.x, sum[0]); sum[1] = fmaf(f1, x.y, sum[1]);
          sum[2] = fmaf(f0, x.z, sum[2]); sum[3] = fmaf(f1, x.w, sum[3]);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int q = q0 + n * 8 + t4 * 2 + x;
          if (q >= nq) continue;
          const int j = quotient16(q, a.group_inv), h = seg.kvh * group + q - j * group;
          const float f = !whole ? 1.f : seg.len < 0 ? 0.f : result_scale(a, pos[n][x], den[x]);
          float *to = whole ? a.out + (((long long)seg.b * a.c + j) * a.hq + h) * HD : part + (q - q0) * HD;
          to[d * 16 + g4] = sum[x] * f;
          to[d * 16 + g4 + 8] = sum[x + 2] * f;
          if (!whole && d == 0 && g4 == 0) ml_cta[q - q0] = make_float2(M[x], den[x]);
        }
      }
    }
    break;
  }
  if (LINE) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    return;
  }
  if (gridDim.x == 1) return;
  const int q0 = seg.qg * Q;
  join_cluster<HD>(a, seg, q0, min(Q, nq - q0), base, smem_u32(ml_cta), C::kThreads);
}

// ------------------------------------------------------------------------------------ host side
template <int HD, int QN>
cudaError_t launch_mma(const PagedAttnArgs &a, const PagedPlan &plan, cudaStream_t st) {
  constexpr int W = kPagedWarps, M = kMoreWarps;
  static bool done[2][kMaxDevices] = {}, more_done[kMaxDevices] = {};
  if (plan.ctas == 0 && plan.workers == kSms * M)
    return launch_line<HD, 8 * QN, kKeys>(a, plan, paged_mma_kernel<HD, QN, M, true>, PagedCfg<HD, M>::kSmem, more_done, st);
  return launch_units<HD, 8 * QN, kKeys>(a, plan, paged_mma_kernel<HD, QN, W, true>, paged_mma_kernel<HD, QN, W, false>, PagedCfg<HD, W>::kSmem, done, st);
}
template <int HD>
cudaError_t launch_hd(const PagedAttnArgs &a, const PagedPlan &plan, cudaStream_t st) {
  return plan.queries == 8 ? launch_mma<HD, 1>(a, plan, st) : launch_mma<HD, 2>(a, plan, st);
}

}  // namespace

cudaError_t launch_paged_attn(PagedAttnArgs a, const PagedPlan &plan, int dtype, int hd, cudaStream_t st) {
  const int es = dtype == FC_F32 ? 4 : 2;
  a.hd = hd; a.elem_bytes = es;
  a.page_bytes = a.pool.page_stride * es; a.head_bytes = a.pool.head_stride * es; a.slot_bytes = a.pool.slot_stride * es;
  if (plan.kind == kFma) return launch_paged_fma(a, plan, hd, st);
  if (plan.kind == kUmma) return launch_paged_umma(a, hd, st);
  return hd == 128 ? launch_hd<128>(a, plan, st) : hd == 64 ? launch_hd<64>(a, plan, st) : launch_hd<32>(a, plan, st);
}

}  // namespace fc
