// Window attention over pages for many queries per kv head (windows of rows on grouped heads), on tcgen05: bf16, hd 64 / 128.
//
// A unit is a kv head of a sequence and 128 queries, the rows of the MMAs: S = Q.K^T (128 x 64 keys) and O = P.V (128 x hd), both operands
// of the first and V of the second in shared memory, P in tensor memory.  The line of tiles, here of 64 keys, and the joining of parts are those of
// k_paged_attn.cu.  One CTA per SM, three groups of four warps:
//   softmax (two groups): the groups take turns at the tiles.  A thread owns a query: its scores come out of tensor memory in one piece, so that maximum
//     and sum need no exchange; probabilities go back as three bf16 parts (all 24 bits), and the product of a tile is added to the thread's output in
//     fp32 (the tensor core's own additions are not rounded to nearest), a tile later, when it has long been there.  While one group does
//     this the tensor core works for the other.  Where a segment ends, the groups join through shared memory.
//   the third: a warp issues the first product, one the second; two load tiles, keys and values by TMA, a box per page and sub-tile (pages of
//     whole groups of eight slots), or in turn by cp.async (any other page), and the queries of a unit in front of its first tile (by TMA with the
//     keys where the heads of a group divide 128: the keys' warp runs tiles ahead, and a box of them is here sooner than 128 rows of copies).
// Measured (hd 64, 16 sequences x 4 kv heads x 128 queries, 3640 keys on average): 34.9 us with the join, 0.22 PFLOP/s, or 0.44 with the parts; K/V at 1.75 TB/s.  Bound by the
// latency of the softmax: two warps per scheduler issue in 40 % of the cycles, the tensor pipe is 20 % busy.
// Spills, in bytes stored and loaded: 324 and 300 at hd 64, 564 and 600 at hd 128 by TMA; 308 and 272, 516 and 544 by copies.  (Compiled without the code for tiles
// that some row does not see whole 184 and 188, 440 and 508 by TMA; without the third group none: 168 registers are what all threads start with.)
// Every wait is bounded: where one runs out the CTA says so in its status word, and the joining kernel writes NaN for what it was to compute.
#include <type_traits>

#include "fc_paged.cuh"
#include "fc_plan.h"

namespace fc {

namespace {

constexpr int kKeys = kUmmaKeys, kQueries = kUmmaQueries;
constexpr int kThreads = 384;

template <int HD>
struct UmmaCfg {
  static constexpr int SUB = HD / 64;                              // sub-tiles of 64 elements (128 bytes a row)
  static constexpr uint32_t kSub = kKeys * 128u, kHalf = SUB * kSub, kTile = 2 * kHalf;
  static constexpr int S = HD == 64 ? 8 : 4;                       // 128 KB of tiles
  static constexpr uint32_t kQSub = kQueries * 128u, kQ = SUB * kQSub;
  static constexpr uint32_t kExchange = kQueries * 64 * 4;         // 64 columns of the output at a time
  // tensor memory of a group, 256 columns: scores, the parts of P, the product.  At hd 128 the parts lie over the scores, so that the next scores
  // follow the product; at hd 64 they can be made before it.
  static constexpr bool kApart = HD == 64;
  static constexpr uint32_t kP = kApart ? 64 : 0, kO = kApart ? 160 : 128;
  static constexpr size_t kSmem = 1024 + (size_t)S * kTile + 2 * kQ + kExchange;
  // Registers a thread, of softmax and of the third group: 384 x 168 in all, what the launch holds.  (hd 64, 16 sequences of 16 rows: 224 and 56 35.7 us,
  // 208 and 88 35.0, 200 and 104 36.3; hd 128, 8 x 8 x 128 queries over 2000 keys: 45.2, 49.2 with 208 and 88.)
  static constexpr int kSoftRegs = HD == 64 ? 208 : 224, kLoadRegs = HD == 64 ? 88 : 56;
  static_assert(256 * kSoftRegs + 128 * kLoadRegs == kThreads * 168, "");
};

// 16-byte piece `ch` of row `r` in a tile of `rows` rows: rows of 128 bytes, the 128-byte swizzle of the MMA's operands.
__device__ __forceinline__ uint32_t uoff(int rows, int r, int ch) {
  return (uint32_t)(ch >> 3) * (uint32_t)rows * 128u + (uint32_t)r * 128u + (uint32_t)(((ch & 7) ^ (r & 7)) << 4);
}
// V as the B operand [hd x keys]: elements (N) adjacent, blocks of 64 of them a sub-tile apart, groups of eight keys 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_v(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((kKeys * 128u) >> 4) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.b32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r != 0;
}
// A in tensor memory
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}
// Columns of this thread's lane.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float *v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, float *v) {
  uint32_t r[64];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
      : "r"(taddr) : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 64; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)), "l"(*reinterpret_cast<unsigned long long *>(&c)));
  return *reinterpret_cast<float2 *>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<unsigned long long *>(&a)), "l"(*reinterpret_cast<unsigned long long *>(&b)));
  return *reinterpret_cast<float2 *>(&r);
}
__device__ __forceinline__ void load_4d(uint32_t dst, const CUtensorMap *map, const int (&x)[4], uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(bar) : "memory");
}

// Tensor maps of keys and values: dimension 0 are the elements; which of 1 .. 3 are slots, heads and pages.  box: slots that one load takes.
// Of the queries: elements, heads of a group, rows, kv heads, a unit per box, where the heads of a group divide 128 (q_rows: window rows of a box;
// 0: the queries are copied by a warp).
struct PageMaps {
  CUtensorMap k, v, q;
  int slot_dim, head_dim, page_dim, box, q_rows;
};

template <int HD, bool TMA>
__global__ void __launch_bounds__(kThreads, 1) paged_umma_kernel(const __grid_constant__ PageMaps maps, const __grid_constant__ PagedAttnArgs a) {
  using C = UmmaCfg<HD>;
  constexpr int S = C::S, PER = HD / 8;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) unsigned long long k_full[S], v_full[S], k_empty[S], v_empty[S], q_full[2], q_free[2], s_ready[2], s_free[2], p_ready[2], o_ready[2], ex_full, ex_free,
      drained[2], odd_bar[2], tmem_here;
  __shared__ unsigned int tmem_base_s, bad_keys[S][2], odd_keys[2][2];
  __shared__ int gave_up;
  __shared__ float2 ml[kQueries];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char *base_g = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t q_base = base + S * C::kTile;
  float4 *exchange = reinterpret_cast<float4 *>(base_g + S * C::kTile + 2 * C::kQ);      // piece c4 of row r at r * 16 + (c4 ^ (r & 15))

  if (tid < S) {
    mbar_init(smem_u32(&k_full[tid]), 1); mbar_init(smem_u32(&v_full[tid]), 1); mbar_init(smem_u32(&k_empty[tid]), 1); mbar_init(smem_u32(&v_empty[tid]), 1);
    fence_barrier_init();
  } else if (tid >= 32 && tid < 34) {
    const int i = tid - 32;
    mbar_init(smem_u32(&q_full[i]), 1); mbar_init(smem_u32(&q_free[i]), 1); mbar_init(smem_u32(&s_ready[i]), 1); mbar_init(smem_u32(&o_ready[i]), 1);
    mbar_init(smem_u32(&s_free[i]), 128); mbar_init(smem_u32(&p_ready[i]), 128); mbar_init(smem_u32(&odd_bar[i]), 128); mbar_init(smem_u32(&drained[i]), 1);
    odd_keys[i][0] = odd_keys[i][1] = 0u;
    fence_barrier_init();
  } else if (tid == 64) {
    mbar_init(smem_u32(&ex_full), 128); mbar_init(smem_u32(&ex_free), 128); mbar_init(smem_u32(&tmem_here), 1);
    gave_up = 0;
    fence_barrier_init();
  }
  fence_proxy_async();
  Place seg;
  int n_mine;
  if (!my_piece<kKeys, true>(a, blockIdx.x, kSms, seg, n_mine)) return;
  __syncthreads();
  // tensor memory comes while the loads begin; whoever uses it waits for it
  if (warp == 8) {
    tmem_alloc(smem_u32(&tmem_base_s), 512);
    tc_fence_before();
    if (lane == 0) mbar_arrive(smem_u32(&tmem_here));
  }
  volatile int *quit = &gave_up;
  // Where tensor memory begins (group w from column 256 w), to a whole warp; false if it did not come.
  auto tensor_memory = [&](uint32_t &t) {
    if (!mbar_wait_warp(smem_u32(&tmem_here), 0, quit)) return false;
    tc_fence_after();
    t = __shfl_sync(0xffffffffu, *(volatile unsigned int *)&tmem_base_s, 0);
    return true;
  };
  const int group = a.group, nq = a.nq;
  const float sl2 = rsqrtf((float)HD) * 1.4426950408889634f;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kLoadRegs));
    // Barriers of the tiles: what TMA or copies complete, and what the products free.  A warp that gives up a wait leaves its loop.
    auto drain = [&](int k) {                            // what this warp issued has completed, its arrivals are made: then memory may be given up
      if (elect_one()) umma_commit(smem_u32(&drained[k]));
      __syncwarp();
      const unsigned long long t0 = clock64();
      while (!mbar_try(smem_u32(&drained[k]), 0))
        if ((unsigned long long)(clock64() - t0) > kSpinBudget) { *quit = 1; break; }
      __syncwarp();
    };
    // The queries of a unit into buffer `so & 1` (ordinal of the segment), behind the products of the segment that had it before.
    auto load_queries = [&](const Place &at, int so) {
      if (so >= 2 && !mbar_wait_warp(smem_u32(&q_free[so & 1]), (uint32_t)((so >> 1) - 1) & 1u, quit)) return false;
      const uint32_t qb = q_base + (uint32_t)(so & 1) * C::kQ;
      const __nv_bfloat16 *from = (const __nv_bfloat16 *)a.q + (long long)at.b * a.c * a.q_stride + (long long)at.kvh * group * HD;
#pragma unroll 1
      for (int r0 = 0; r0 < kQueries; r0 += 32) {        // a lane's row, then the warp goes over the pieces of 32 rows
        const int q = min(at.qg * kQueries + r0 + lane, nq - 1), j = quotient16(q, a.group_inv);
        const long long off = j * a.q_stride + (q - j * group) * HD;
#pragma unroll 4
        for (int y = 0; y < PER; ++y) {
          const int r = y * (32 / PER) + lane / PER;
          copy16(qb + uoff(kQueries, r0 + r, lane % PER), from + __shfl_sync(0xffffffffu, off, r) + (lane % PER) * 8, 16u);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&q_full[so & 1]));
      return true;
    };
    // The two warps that issue MMAs run as one, on values that are broadcast from their first lane, and one thread is elected to issue:
    // descriptors are then worked out once in uniform registers.  (Inside `if (lane == 0)` an MMA cost the issuing thread about 60 cycles.)
    const uint32_t tiles = __shfl_sync(0xffffffffu, base, 0);
    const int n_all = __shfl_sync(0xffffffffu, n_mine, 0);
    if (warp == 8) {
      // ------------------------------------------------------------------------------------------ S = Q.K^T
      constexpr uint32_t id_s = make_idesc(kKeys);
      int so = 0, left = min(n_all, seg.k.n - seg.t);    // ordinal of the segment, its tiles that are left
      Place at = seg;
      bool first = true;
      uint32_t tm = 0;
      const bool got = tensor_memory(tm);
      for (int i = 0; got && i < n_all; ++i) {
        const int st = i % S, w = i & 1;
        if (first && !mbar_wait_warp(smem_u32(&q_full[so & 1]), (uint32_t)(so >> 1) & 1u, quit)) break;
        if (!mbar_wait_warp(smem_u32(&k_full[st]), (uint32_t)(i / S) & 1u, quit)) break;
        // the scores' place: read (hd 64), or the product of the parts over it done (hd 128)
        if (i >= 2 && !mbar_wait_warp(smem_u32(C::kApart ? &s_free[w] : &o_ready[w]), (uint32_t)((i - 2) >> 1) & 1u, quit)) break;
        tc_fence_after();
        const uint64_t qd = smem_desc_sw128(tiles + S * C::kTile + (uint32_t)(so & 1) * C::kQ), kd = smem_desc_sw128(tiles + st * C::kTile);
        const bool last = --left == 0;
        if (elect_one()) {
#pragma unroll
          for (int ks = 0; ks < HD / 16; ++ks)           // descriptors count in 16 bytes
            umma_bf16(tm + w * 256, qd + ((ks >> 2) * C::kQSub + (ks & 3) * 32) / 16, kd + ((ks >> 2) * C::kSub + (ks & 3) * 32) / 16, id_s, ks > 0);
          umma_commit(smem_u32(&s_ready[w]));
          umma_commit(smem_u32(&k_empty[st]));
          if (last) umma_commit(smem_u32(&q_free[so & 1]));
        }
        __syncwarp();
        first = last;
        if (last && i + 1 < n_all) {
          ++so;
          move_on<kKeys>(a, at, min(n_all, at.k.n - at.t));
          left = __shfl_sync(0xffffffffu, min(n_all - i - 1, at.k.n - at.t), 0);
        }
      }
      drain(0);
    } else if (warp == 11) {
      // ------------------------------------------------------------------------------------------ O = P.V
      constexpr uint32_t id_o = make_idesc(HD) | (1u << 16);       // V: N adjacent
      uint32_t tm = 0;
      const bool got = tensor_memory(tm);
      for (int i = 0; got && i < n_all; ++i) {
        const int st = i % S, w = i & 1;
        if (!mbar_wait_warp(smem_u32(&v_full[st]), (uint32_t)(i / S) & 1u, quit)) break;
        if (!mbar_wait_warp(smem_u32(&p_ready[w]), (uint32_t)(i >> 1) & 1u, quit)) break;
        tc_fence_after();
        const uint64_t vd = desc_v(tiles + st * C::kTile + C::kHalf);
        if (elect_one()) {
#pragma unroll
          for (int part = 2; part >= 0; --part)
#pragma unroll
            for (int ks = 0; ks < kKeys / 16; ++ks)
              umma_bf16_ts(tm + w * 256 + C::kO, tm + w * 256 + C::kP + part * 32 + ks * 8, vd + ks * 128, id_o, part < 2 || ks > 0);
          umma_commit(smem_u32(&o_ready[w]));
          umma_commit(smem_u32(&v_empty[st]));
        }
        __syncwarp();
      }
      drain(1);
    } else if (TMA) {
      // ------------------------------------------------------------------------------------------ tiles by TMA, keys by one warp, values by the other
      const bool keys = warp == 9;
      unsigned long long *full = keys ? k_full : v_full, *empty = keys ? k_empty : v_empty;
      const CUtensorMap *map = keys ? &maps.k : &maps.v;
      Place ld = seg;
      const int boxes = kKeys / maps.box, ahead = 32 / boxes;      // boxes of a tile; tiles whose pages the lanes look up at once
      bool ok = true;
      int i = 0, st = 0, asked = 0;                      // asked: units whose queries this warp requested
      uint32_t turn = 1;                                 // parity of the wait for an empty stage: none is waited for the first time round
      for (int so = 0; i < n_all && ok; ++so) {          // segment by segment
        const int seg_n = min(n_all - i, ld.k.n - ld.t);
        const int see_from = window_first(ld.len + quotient16(ld.qg * kQueries, a.group_inv), a.window);
        const int see_to = min(ld.len + quotient16(min(nq - 1, ld.qg * kQueries + kQueries - 1), a.group_inv), a.cap - 1);
        for (int g0 = 0; g0 < seg_n && ok; g0 += ahead) {
          const int t = tile_key(ld.k, ld.t + g0 + lane / boxes, kKeys) + lane % boxes * maps.box;
          int page = -2, x[3] = {0, 0, 0};               // the lane's box: -2, no row sees it, it is not loaded; -1: nor one without a page
          if (g0 + lane / boxes < seg_n && t <= see_to && (t + maps.box > see_from || t < a.n_sink)) {
            const int e = (int)((unsigned int)t / (unsigned int)a.pool.page_size), slot = t - e * a.pool.page_size;
            page = max(-1, a.table[(long long)ld.b * a.width + e]);
            if (page >= a.pool.n_pages) page = -1;
#pragma unroll
            for (int d = 0; d < 3; ++d) x[d] = d + 1 == maps.slot_dim ? slot : d + 1 == maps.head_dim ? ld.kvh : page;
          }
          if (g0 == 0) {                                 // the queries first, the table is still on its way
            if (maps.q_rows && keys) {
              if (so >= 2 && !mbar_wait_warp(smem_u32(&q_free[so & 1]), (uint32_t)((so >> 1) - 1) & 1u, quit)) { ok = false; break; }
              const uint32_t bar = smem_u32(&q_full[so & 1]), dst = tiles + S * C::kTile + (uint32_t)(so & 1) * C::kQ;
              if (elect_one()) {
                mbar_expect_tx(bar, C::kQ);
#pragma unroll
                for (int k = 0; k < C::SUB; ++k) {
                  const int y[4] = {k * 64, 0, (a.first + ld.b) * a.c + ld.qg * maps.q_rows, ld.kvh};
                  load_4d(dst + k * C::kQSub, &maps.q, y, bar);
                }
              }
              __syncwarp();
              ++asked;
            } else if (!maps.q_rows && !keys && !load_queries(ld, so)) {
              ok = false;
              break;
            }
          }
          const unsigned int all_bad = __ballot_sync(0xffffffffu, page == -1), all_here = __ballot_sync(0xffffffffu, page >= 0);
          const unsigned int of_tile = (1u << boxes) - 1;
          const int n = min(ahead, seg_n - g0);
          for (int g = 0; g < n; ++g, ++i) {
            const unsigned int here = all_here >> (g * boxes) & of_tile;
            if (i >= S && !mbar_wait_warp(smem_u32(&empty[st]), turn, quit)) { ok = false; break; }
            const uint32_t bar = smem_u32(&full[st]), dst = tiles + st * C::kTile + (keys ? 0u : C::kHalf);
            if (!keys && lane == 0) {
              unsigned long long gone = 0;
              for (unsigned int bad = all_bad >> (g * boxes) & of_tile; bad; bad &= bad - 1) gone |= (~0ull >> (64 - maps.box)) << ((__ffs(bad) - 1) * maps.box);
              bad_keys[st][0] = (unsigned int)gone;
              bad_keys[st][1] = (unsigned int)(gone >> 32);
            }
            if (lane == 0) mbar_expect_tx(bar, (uint32_t)(__popc(here) * maps.box) * (HD * 2u));
            __syncwarp();
            for (int b = 0; b < boxes; ++b) {
              const int from = g * boxes + b;
              const int at[4] = {0, __shfl_sync(0xffffffffu, x[0], from), __shfl_sync(0xffffffffu, x[1], from), __shfl_sync(0xffffffffu, x[2], from)};
              if ((here >> b & 1u) && elect_one()) {
#pragma unroll
                for (int k = 0; k < C::SUB; ++k) {
                  const int y[4] = {k * 64, at[1], at[2], at[3]};
                  load_4d(dst + (uint32_t)(b * maps.box) * 128u + k * C::kSub, map, y, bar);
                }
              }
            }
            if (++st == S) { st = 0; turn ^= 1u; }
          }
        }
        if (i < n_all) move_on<kKeys>(a, ld, seg_n);
      }
      if (i < n_all) {                                   // gave up: wait (bounded) for what was requested
        const unsigned long long t0 = clock64();
        for (int k = 0; k < S && k < i; ++k)
          while (!mbar_try(smem_u32(&full[k]), last_copy_parity(i, S, k)))
            if ((unsigned long long)(clock64() - t0) > kSpinBudget / 4) break;
        for (int k = 0; k < 2 && k < asked; ++k)
          while (!mbar_try(smem_u32(&q_full[k]), last_copy_parity(asked, 2, k)))
            if ((unsigned long long)(clock64() - t0) > kSpinBudget / 4) break;
      }
    } else {
      // ------------------------------------------------------------------------------------------ tiles by cp.async, two warps in turn
      const int lw = warp - 9;
      Place ld = seg;
      int pending = -1, so = -1;
      bool ok = true;
      auto landed = [&]() {                              // the copies of `pending` are here: for the tensor core to read
        if (pending < 0) return;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) { mbar_arrive(smem_u32(&k_full[pending])); mbar_arrive(smem_u32(&v_full[pending])); }
        pending = -1;
      };
      // a wait in front of which the copies on their way are handed over: what waits for them may be what it waits for
      auto wait_for = [&](uint32_t bar, uint32_t parity) {
        if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        landed();
        return mbar_wait_warp(bar, parity, quit);
      };
      bool begins = true;                                // tile i is the first of a segment
      for (int i = 0, on; i < n_mine; i += on, begins = i < n_mine && move_on<kKeys>(a, ld, on) > 0) {
        so += begins;
        if (begins && lw == query_copier(i)) {           // always the same warp, whose tile it is or not
          asm volatile("cp.async.wait_group 0;" ::: "memory");
          landed();                                      // the products that the wait is for may need them
          if (!load_queries(ld, so)) { ok = false; break; }
        }
        on = 1;
        if (i % kCopyWarps != lw) continue;
        if (ld.t + kCopyWarps < ld.k.n) on = kCopyWarps; // nothing begins at the other warp's tile
        const int st = i % S;
        // ---- pages of the lanes' keys (lane, lane + 32)
        const int see_from = window_first(ld.len + quotient16(ld.qg * kQueries, a.group_inv), a.window);
        const int see_to = min(ld.len + quotient16(min(nq - 1, ld.qg * kQueries + kQueries - 1), a.group_inv), a.cap - 1);
        long long off[2];
        unsigned int bad[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int t = tile_key(ld.k, ld.t, kKeys) + x * 32 + lane;
          const bool seen = t <= see_to && (t >= see_from || t < a.n_sink);
          off[x] = -1;
          bool missing = false;
          if (seen) {
            const int e = (int)((unsigned int)t / (unsigned int)a.pool.page_size), page = a.table[(long long)ld.b * a.width + e];
            missing = page < 0 || page >= a.pool.n_pages;
            if (!missing) off[x] = (long long)page * a.page_bytes + (long long)(t - e * a.pool.page_size) * a.slot_bytes;
          }
          bad[x] = __ballot_sync(0xffffffffu, missing);
        }
        if (i >= S && (!wait_for(smem_u32(&k_empty[st]), (uint32_t)(i / S - 1) & 1u) || !wait_for(smem_u32(&v_empty[st]), (uint32_t)(i / S - 1) & 1u))) {
          ok = false;
          break;
        }
        if (lane == 0) { bad_keys[st][0] = bad[0]; bad_keys[st][1] = bad[1]; }
        const char *k0 = (const char *)a.pool.k + ld.kvh * a.head_bytes + (lane % PER) * 16;
        const char *v0 = (const char *)a.pool.v + ld.kvh * a.head_bytes + (lane % PER) * 16;
        const uint32_t kb = base + st * C::kTile;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll 4
          for (int y = 0; y < PER; ++y) {
            const int r = y * (32 / PER) + lane / PER;
            const long long o = __shfl_sync(0xffffffffu, off[x], r);
            const uint32_t d = kb + uoff(kKeys, x * 32 + r, lane % PER), bytes = o < 0 ? 0u : 16u;      // keys that no row sees become zeros
            copy16(d, k0 + (o < 0 ? 0 : o), bytes);
            copy16(d + C::kHalf, v0 + (o < 0 ? 0 : o), bytes);
          }
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        landed();
        pending = st;
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      if (ok) landed();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftRegs));
    // -------------------------------------------------------------------------------------------- softmax
    const int w = warp >> 2, row = tid & 127;
    uint32_t sc = 0;
    bool ok = tensor_memory(sc);
    sc += w * 256 + ((uint32_t)(warp & 3) << 21);          // this warp's 32 lanes
    int i = w, done = 0, exchanges = 0;
    uint32_t odd_phase = 0;
    while (ok) {
      const int seg_n = min(n_mine - done, seg.k.n - seg.t);
      const int q0 = seg.qg * kQueries, q = q0 + row, qc = min(q, nq - 1), j = quotient16(qc, a.group_inv), h = seg.kvh * group + qc - j * group;
      const int pos = seg.len + j, low = window_first(pos, a.window);
      const int p_first = seg.len + quotient16(q0, a.group_inv), p_last = seg.len + quotient16(min(nq - 1, q0 + kQueries - 1), a.group_inv);
      const int low_last = window_first(p_last, a.window);
      float m = -INFINITY, l = 0.f, corr = 1.f;          // corr: what the output so far counts once the last tile's product is added
      int last = -1;                                     // the tile whose product is not added yet
      float2 o[HD / 2];
#pragma unroll
      for (int c = 0; c < HD / 2; ++c) o[c] = make_float2(0.f, 0.f);
      // O = corr O + P.V of the last tile
      auto add_product = [&]() {
        if (last < 0) return;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&o_ready[w]), (uint32_t)(last >> 1) & 1u, quit));
        if (!ok) return;
        tc_fence_after();
        const float2 f = make_float2(corr, corr);
#pragma unroll
        for (int c0 = 0; c0 < HD / 2; c0 += 16) {
          float y[32];
          tmem_ld32(sc + C::kO + c0 * 2, y);
#pragma unroll
          for (int c = 0; c < 16; ++c) o[c0 + c] = fma2(o[c0 + c], f, make_float2(y[2 * c], y[2 * c + 1]));
        }
        tc_fence_before();
      };
      for (; i < done + seg_n; i += 2) {
        const int st = i % S;
        const uint32_t turn = (uint32_t)(i >> 1) & 1u;
        const int key0 = tile_key(seg.k, seg.t + i - done, kKeys);
        // the scores, and the values with what their loader wrote beside them (the keys' stage may be another tile's by now: it is free when
        // the scores are made; the values' is not before the probabilities have been used)
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&s_ready[w]), turn, quit) && mbar_wait(smem_u32(&v_full[st]), (uint32_t)(i / S) & 1u, quit));
        if (!ok) break;
        tc_fence_after();
        // Before the scores are loaded: at hd 128 they lie over parts that the product still reads, and so the registers hold one or the other (behind the
        // exponentials, at hd 64, 38.2 us against 36.8 on 16 sequences of 16 rows; in front of the wait above 37.4).
        add_product();
        if (!ok) break;
        const unsigned int bad0 = bad_keys[st][0], bad1 = bad_keys[st][1];
        const bool masked = key0 + kKeys - 1 > p_first || (key0 < low_last && key0 + kKeys > a.n_sink) || (bad0 | bad1);
        // Tiles that all rows see whole are most of them and have code of their own, without the jumps over what the others need.
        auto tile = [&](auto kind) {
        constexpr bool hard = decltype(kind)::value;
        float s[kKeys];
        tmem_ld64(sc, s);
        if (C::kApart) {
          tc_fence_before();
          mbar_arrive(smem_u32(&s_free[w]));
        }
        if (hard) {
          // bit k: whether the row sees key key0 + k (all up to `to` but those between the sinks and the window), and has a page for it
          auto below = [](int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; };     // bits 0 .. n - 1
          const unsigned long long see = below(pos + 1 - key0) & ~(below(low - key0) & ~below(a.n_sink - key0));
          const unsigned int see0 = (unsigned int)see, see1 = (unsigned int)(see >> 32);
          if (bad0 | bad1) {
#pragma unroll
            for (int k = 0; k < kKeys; ++k)
              if ((k < 32 ? bad0 >> k : bad1 >> (k - 32)) & 1u) s[k] = quiet_nan();
          }
#pragma unroll
          for (int k = 0; k < kKeys; ++k)
            if (!((k < 32 ? see0 >> k : see1 >> (k - 32)) & 1u)) s[k] = -INFINITY;
        }
        float mx[4] = {fmaxf(m, s[0]), s[1], s[2], s[3]};
#pragma unroll
        for (int k = 4; k < kKeys; k += 8)
#pragma unroll
          for (int x = 0; x < 4; ++x) mx[x] = k + 4 + x < kKeys ? fmaxf(fmaxf(mx[x], s[k + x]), s[k + 4 + x]) : fmaxf(mx[x], s[k + x]);
        mx[0] = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        float corr_now = mx[0] == m ? 1.f : ex2((m - mx[0]) * sl2);                            // first tile: 2^-inf = 0
        const float l_corr = corr_now;
        m = mx[0];
        const float mb = m == -INFINITY ? 0.f : -m * sl2;
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        auto exponentials = [&](int from) {              // of 16 scores
#pragma unroll
          for (int k = from; k < from + 16; k += 2) {
            const float2 x = fma2(make_float2(s[k], s[k + 1]), make_float2(sl2, sl2), make_float2(mb, mb));
            s[k] = ex2(x.x);
            s[k + 1] = ex2(x.y);
            sum[(k >> 1) & 1] = add2(sum[(k >> 1) & 1], make_float2(s[k], s[k + 1]));
          }
        };
        // values that are not finite, in a tile that some row does not see whole (by TMA its unseen slots hold anything): those keys are
        // added row by row and taken out of the tile (a probability of zero would carry them to rows that do not see them)
        if (hard) {
#pragma unroll
          for (int from = 0; from < kKeys; from += 16) exponentials(from);
          const uint32_t vb = base + st * C::kTile + C::kHalf;
          unsigned char *vg = base_g + (vb - base);
          unsigned int odd0 = 0, odd1 = 0;
          for (int e = row; e < kKeys * PER; e += 128) {
            const int r = e / PER;
            const uint4 x = *reinterpret_cast<const uint4 *>(vg + uoff(kKeys, r, e % PER));
            const uint32_t y[4] = {x.x, x.y, x.z, x.w};
            bool found = false;
#pragma unroll
            for (int c = 0; c < 4; ++c) found |= (y[c] & 0x7f80u) == 0x7f80u || (y[c] & 0x7f800000u) == 0x7f800000u;
            if (found) { if (r < 32) odd0 |= 1u << r; else odd1 |= 1u << (r - 32); }
          }
          if (odd0) atomicOr(&odd_keys[w][0], odd0);
          if (odd1) atomicOr(&odd_keys[w][1], odd1);
          mbar_arrive(smem_u32(&odd_bar[w]));
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&odd_bar[w]), odd_phase, quit));
          if (!ok) return;
          odd_phase ^= 1u;
          odd0 = *(volatile unsigned int *)&odd_keys[w][0];
          odd1 = *(volatile unsigned int *)&odd_keys[w][1];
          if (odd0 | odd1) {
            bool scaled = false;                         // rows that see none of them are computed as ever: what they hold may be left over from anything
#pragma unroll 1
            for (unsigned long long left = ((unsigned long long)odd1 << 32) | odd0; left; left &= left - 1) {
              const int kk = __ffsll((long long)left) - 1;
              if (!sees(pos, key0 + kk, a.window, a.n_sink)) continue;
              if (!scaled) {
#pragma unroll
                for (int c = 0; c < HD / 2; ++c) { o[c].x *= corr_now; o[c].y *= corr_now; }
                corr_now = 1.f;
                scaled = true;
              }
              float p = 0.f;
#pragma unroll
              for (int k = 0; k < kKeys; ++k)
                if (k == kk) p = s[k];
#pragma unroll
              for (int ch = 0; ch < PER; ++ch) {
                const uint4 x = *reinterpret_cast<const uint4 *>(vg + uoff(kKeys, kk, ch));
                const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                  o[ch * 4 + c].x = fmaf(p, low_half(y[c]), o[ch * 4 + c].x);
                  o[ch * 4 + c].y = fmaf(p, high_half(y[c]), o[ch * 4 + c].y);
                }
              }
            }
            mbar_arrive(smem_u32(&odd_bar[w]));
            ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&odd_bar[w]), odd_phase, quit));
            if (!ok) return;
            odd_phase ^= 1u;
            for (int e = row; e < kKeys * PER; e += 128) {
              const int r = e / PER;
              if ((r < 32 ? odd0 >> r : odd1 >> (r - 32)) & 1u) *reinterpret_cast<uint4 *>(vg + uoff(kKeys, r, e % PER)) = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async();
            if (row == 0) odd_keys[w][0] = odd_keys[w][1] = 0u;
          }
        }
        corr = corr_now;
        last = i;
        // ---- probabilities in three parts, cut off (8 bits each), 16 keys at a time: what is between exponentials overlaps with them
#pragma unroll
        for (int from = 0; from < kKeys; from += 16) {
          if (!hard) exponentials(from);
#pragma unroll
          for (int part = 0; part < 3; ++part) {
            uint32_t r[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              float &p0 = s[from + 2 * k], &p1 = s[from + 2 * k + 1];
              r[k] = __byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x7632);
              if (part < 2) {
                const float2 x = fma2(make_float2(low_half(r[k]), high_half(r[k])), make_float2(-1.f, -1.f), make_float2(p0, p1));
                p0 = x.x;
                p1 = x.y;
              }
            }
            tmem_st8(sc + C::kP + part * 32 + from / 2, r);
          }
        }
        sum[0] = add2(sum[0], sum[1]);
        l = fmaf(l, l_corr, sum[0].x + sum[0].y);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        };
        if (masked) tile(std::true_type());
        else tile(std::false_type());
        if (!ok) break;
        mbar_arrive(smem_u32(&p_ready[w]));
      }
      if (ok) add_product();
      if (!ok) break;
      // ---- the groups' results: the second hands over, the first adds up and writes
      const bool whole = seg_n == seg.k.n;
      float *part = a.parts + ((long long)blockIdx.x * 2 + (done > 0)) * part_floats(kQueries, HD);
      float *to = whole ? a.out + (((long long)seg.b * a.c + j) * a.hq + h) * HD : part + row * HD;
#pragma unroll
      for (int c0 = 0; c0 < HD / 2; c0 += 32, ++exchanges) {
        if (w == 1) {
          if (exchanges > 0) ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&ex_free), (uint32_t)(exchanges - 1) & 1u, quit));
          if (!ok) break;
          if (c0 == 0) ml[row] = make_float2(m, l);
#pragma unroll
          for (int c = 0; c < 16; ++c) exchange[row * 16 + (c ^ (row & 15))] = make_float4(o[c0 + 2 * c].x, o[c0 + 2 * c].y, o[c0 + 2 * c + 1].x, o[c0 + 2 * c + 1].y);
          mbar_arrive(smem_u32(&ex_full));
        } else {
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&ex_full), (uint32_t)exchanges & 1u, quit));
          if (!ok) break;
          const float2 other = ml[row];
          const float M = fmaxf(m, other.x), f0 = part_weight(make_float2(m, l), M, sl2), f1 = part_weight(other, M, sl2);
          const float den = fmaf(l, f0, other.y * f1), f = whole ? result_scale(a, pos, den) : 1.f;
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const float4 x = exchange[row * 16 + (c ^ (row & 15))];
            const float4 y = make_float4(fmaf(f1, x.x, f0 * o[c0 + 2 * c].x) * f, fmaf(f1, x.y, f0 * o[c0 + 2 * c].y) * f,
                                         fmaf(f1, x.z, f0 * o[c0 + 2 * c + 1].x) * f, fmaf(f1, x.w, f0 * o[c0 + 2 * c + 1].y) * f);
            if (q < nq) *reinterpret_cast<float4 *>(to + c0 * 2 + 4 * c) = y;
          }
          if (!whole && c0 == 0 && q < nq) *reinterpret_cast<float2 *>(part + kQueries * HD + row * 2) = make_float2(M, den);
          mbar_arrive(smem_u32(&ex_free));
        }
      }
      done += seg_n;
      if (done == n_mine) break;
      move_on<kKeys>(a, seg, seg_n);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 8) tmem_dealloc(*(volatile unsigned int *)&tmem_base_s, 512);
  if (tid == 0) a.status[blockIdx.x] = gave_up != 0;
}

// Maps of one layer's pages, dimensions by stride; false where TMA cannot load them (pages that are not whole groups of eight slots).
using EncodeTiledFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                   const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
bool page_maps(const PagedAttnArgs &a, int hd, PageMaps *maps) {
  if (a.pool.page_size % 8) return false;
  static const EncodeTiledFn enc = [] {
    void *sym = nullptr;
    cudaDriverEntryPointQueryResult qres;
    return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &qres) == cudaSuccess && qres == cudaDriverEntryPointSuccess
               ? (EncodeTiledFn)sym : (EncodeTiledFn) nullptr;
  }();
  if (!enc) return false;
  int box = 64;
  while (a.pool.page_size % box) box /= 2;
  struct Dim { int kind; cuuint64_t n; long long stride; } d[3] = {{0, (cuuint64_t)a.pool.page_size, a.slot_bytes}, {1, (cuuint64_t)a.pool.n_kv_heads, a.head_bytes},
                                                                   {2, (cuuint64_t)a.pool.n_pages, a.page_bytes}};
  for (Dim &x : d)
    if (x.n == 1) x.stride = hd * 2;                     // its stride says nothing
  for (int i = 0; i < 2; ++i)
    for (int k = 0; k < 2 - i; ++k)
      if (d[k].stride > d[k + 1].stride) { const Dim t = d[k]; d[k] = d[k + 1]; d[k + 1] = t; }
  cuuint64_t gdim[4] = {(cuuint64_t)hd, d[0].n, d[1].n, d[2].n}, gstr[3] = {(cuuint64_t)d[0].stride, (cuuint64_t)d[1].stride, (cuuint64_t)d[2].stride};
  cuuint32_t boxes[4] = {64, 1, 1, 1}, ones[4] = {1, 1, 1, 1};
  maps->box = box;
  for (int i = 0; i < 3; ++i) {
    if (gstr[i] >= (1ull << 40)) return false;
    if (d[i].kind == 0) { maps->slot_dim = i + 1; boxes[i + 1] = (cuuint32_t)box; }
    if (d[i].kind == 1) maps->head_dim = i + 1;
    if (d[i].kind == 2) maps->page_dim = i + 1;
  }
  // queries: a box holds the heads of a group for as many rows as make 128 (rows behind a sequence's are another's or zeros: nobody reads their results)
  maps->q_rows = kQueries % a.group ? 0 : kQueries / a.group;
  if (maps->q_rows) {
    cuuint64_t qdim[4] = {(cuuint64_t)hd, (cuuint64_t)a.group, (cuuint64_t)a.batch * a.c, (cuuint64_t)a.pool.n_kv_heads};
    cuuint64_t qstr[3] = {(cuuint64_t)hd * 2, (cuuint64_t)a.q_stride * 2, (cuuint64_t)a.group * hd * 2};
    cuuint32_t qbox[4] = {64, (cuuint32_t)a.group, (cuuint32_t)maps->q_rows, 1};
    if (qstr[1] >= (1ull << 40) ||
        enc(&maps->q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(a.q), qdim, qstr, qbox, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) maps->q_rows = 0;
  }
  for (int v = 0; v < 2; ++v)
    if (enc(v ? &maps->v : &maps->k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, v ? a.pool.v : a.pool.k, gdim, gstr, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) return false;
  return true;
}

template <int HD, bool TMA>
cudaError_t launch(const PageMaps &maps, const PagedAttnArgs &a, cudaStream_t st) {
  using C = UmmaCfg<HD>;
  static bool done[kMaxDevices] = {false};
  const int dev = current_device_slot();
  if (!done[dev]) {
    // the register split is only there to be had if the launch holds what it adds up to
    cudaFuncAttributes at;
    if (cudaError_t e = cudaFuncGetAttributes(&at, paged_umma_kernel<HD, TMA>)) return e;
    if (at.numRegs * kThreads < 256 * C::kSoftRegs + 128 * C::kLoadRegs) return cudaErrorInvalidConfiguration;
    if (cudaError_t e = allow_smem(paged_umma_kernel<HD, TMA>, C::kSmem, done)) return e;
  }
  return by_lines(a, kKeys, [&](const PagedAttnArgs &part) {
    paged_umma_kernel<HD, TMA><<<kSms, kThreads, C::kSmem, st>>>(maps, part);
    if (cudaError_t e = cudaGetLastError()) return e;
    return launch_combine<HD, kQueries, kKeys>(part, kSms, st);
  });
}

}  // namespace

cudaError_t launch_paged_umma(PagedAttnArgs a, int hd, cudaStream_t st) {
  set_groups(a, kQueries);
  a.status = (unsigned int *)a.parts;
  a.parts = (float *)((char *)a.parts + kUmmaStatus);
  PageMaps maps;
  memset(&maps, 0, sizeof maps);
  if (page_maps(a, hd, &maps)) return hd == 128 ? launch<128, true>(maps, a, st) : launch<64, true>(maps, a, st);
  return hd == 128 ? launch<128, false>(maps, a, st) : launch<64, false>(maps, a, st);
}

}  // namespace fc
