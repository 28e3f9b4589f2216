// Paged K/V cache: rotation and K/V write into pages; entry points of the operations on one layer.
#include <climits>
#include <cmath>
#include <cstring>

#include "fc_internal.h"
#include "fc_paged.h"

namespace fc {

namespace {

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t *>(&v);
}
__device__ __forceinline__ void put4(float *p, const float (&v)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void put4(__nv_bfloat16 *p, const float (&v)[4]) {
  *reinterpret_cast<uint2 *>(p) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
}

// ------------------------------------------------------------------------------------------------ store
struct PagedStoreArgs {
  PageView pool;
  const int32_t *table; int width;
  const int32_t *kv_len;
  const float *qkv; long long qkv_stride;
  void *q;
  int c, hq, hd;
  double turns[64];        // theta^(-2i/hd) / (2 pi): rotations of pair i from one position to the next
};

// A block takes some of the heads of a row.  The row's angles come first, one thread per pair: in whole turns an angle is a 64-bit product whose
// integer part is dropped, so that far positions keep their fraction; what is left goes to sincospif.  Then a thread takes four adjacent
// pairs (i, i + hd/2) of one head: 16-byte loads (issued in front of the angles), 8- or 16-byte stores.
// Bound by latency up to some hundred rows, then by instructions: each block of a row works out all its angles in 64 bits, and the others wait for them.  13B
// shape, 256 rows, eight blocks each: 6.5 us (23.6 MB at 3.6 TB/s, of which L2 keeps the writes: 17 % of DRAM's rate, 48 % of the issue slots); 10.2 us with
// the angles computed by every thread for its four pairs.
template <typename T>
__global__ void __launch_bounds__(256) paged_store_kernel(const __grid_constant__ PagedStoreArgs a) {
  __shared__ float2 turn[64];                            // cosine, sine
  const int r = blockIdx.x, b = r / a.c;
  const int cap = a.width * a.pool.page_size, len = a.kv_len[b];
  if (len < 0) return;
  const long long pos = (long long)len + (r - b * a.c);                  // beyond the table: there is no page, q is rotated all the same
  const int half = a.hd >> 1, per_head = half >> 2, hkv = a.pool.n_kv_heads;
  const int u = blockIdx.y * 256 + threadIdx.x, h = u / per_head, i = (u - h * per_head) << 2;
  const bool mine = h < a.hq + 2 * hkv;
  float4 x, y;
  if (mine) {
    const float *src = a.qkv + r * a.qkv_stride + h * a.hd + i;
    x = *reinterpret_cast<const float4 *>(src);
    y = *reinterpret_cast<const float4 *>(src + half);
  }
  const int page = pos < cap ? page_of(a.table + (long long)b * a.width, a.width, (int)pos, a.pool.page_size, a.pool.n_pages) : -1;
  if (threadIdx.x < half) {
    const double t = (double)pos * a.turns[threadIdx.x];
    float sn, cs;
    sincospif((float)(2.0 * (t - rint(t))), &sn, &cs);
    turn[threadIdx.x] = make_float2(cs, sn);
  }
  __syncthreads();
  const bool is_q = h < a.hq, is_k = !is_q && h < a.hq + hkv;
  if (!mine || (!is_q && page < 0)) return;
  float v0[4] = {x.x, x.y, x.z, x.w}, v1[4] = {y.x, y.y, y.z, y.w};
  if (is_q || is_k) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 t = turn[i + k];
      const float o0 = v0[k] * t.x - v1[k] * t.y, o1 = v0[k] * t.y + v1[k] * t.x;
      v0[k] = o0; v1[k] = o1;
    }
  }
  T *dst;
  if (is_q) dst = (T *)a.q + ((long long)r * a.hq + h) * a.hd;
  else dst = (T *)(is_k ? a.pool.k : a.pool.v) + (long long)page * a.pool.page_stride + (pos % a.pool.page_size) * a.pool.slot_stride +
             (long long)(h - a.hq - (is_k ? 0 : hkv)) * a.pool.head_stride;
  put4(dst + i, v0);
  put4(dst + half + i, v1);
}

// ------------------------------------------------------------------------------------------------ arguments
// FC_OK, or why a call's numbers are refused, whatever its pool looks like otherwise.
int shape_ok(int width, int page_size, int hkv, int hd, int batch, int c, int hq) {
  if (width < 1 || page_size < 1 || hkv < 1 || batch < 1 || c < 1 || c > 64 || hq < 1 || hq % hkv) return FC_ERR_ARG;
  if (hd != 32 && hd != 64 && hd != 128) return FC_ERR_SHAPE;
  if (page_too_large(hkv, page_size, hd) || (long long)width * page_size > INT_MAX - 1024 || (long long)batch * c * hq > INT_MAX / 2 || hq > 512) return FC_ERR_CAPACITY;
  return FC_OK;
}
int call_ok(const fc_pages *pages, int layer, const int32_t *table, int width, const int32_t *kv_len, int batch, int c, int hq) {
  if (int rc = pages_ok(pages)) return rc;
  if (!table || !kv_len || layer < 0 || layer >= pages->n_layers) return FC_ERR_ARG;
  return shape_ok(width, pages->page_size, pages->n_kv_heads, pages->head_dim, batch, c, hq);
}

PageView view_of(const fc_pages *p, int layer) {
  PageView v;
  const long long off = layer * p->layer_stride * (p->dtype == FC_F32 ? 4 : 2);
  v.k = (char *)p->k + off; v.v = (char *)p->v + off;
  v.page_stride = p->page_stride; v.head_stride = p->head_stride; v.slot_stride = p->slot_stride;
  v.n_pages = p->n_pages; v.page_size = p->page_size; v.n_kv_heads = p->n_kv_heads;
  return v;
}

// Turns per position of the pairs.  64 powers are a microsecond, so a thread keeps those of the base and head size that it used last.
void rope_turns(float theta, int hd, double *turns) {
  struct Last { float theta; int hd; double turns[64]; };
  static thread_local Last last = {0.f, 0, {0}};
  if (last.theta != theta || last.hd != hd) {
    for (int i = 0; i < hd / 2; ++i) last.turns[i] = std::pow((double)theta, -2.0 * i / hd) / 6.283185307179586476925286766559;
    last.theta = theta; last.hd = hd;
  }
  memcpy(turns, last.turns, sizeof(double) * (hd / 2));
}

}  // namespace
}  // namespace fc

using namespace fc;

extern "C" int fc_op_paged_store(const fc_pages *pages, int32_t layer, const int32_t *table, int32_t table_width, const int32_t *kv_len,
                                 const float *qkv, int64_t qkv_stride, void *q_out, int32_t batch, int32_t c, int32_t n_heads,
                                 float rope_theta, void *cuda_stream) {
  if (int rc = call_ok(pages, layer, table, table_width, kv_len, batch, c, n_heads)) return rc;
  const int hd = pages->head_dim;
  if (!qkv || !q_out || ((uintptr_t)qkv | (uintptr_t)q_out) % 16 || qkv_stride % 4 ||
      qkv_stride < (int64_t)(n_heads + 2 * pages->n_kv_heads) * hd || !(rope_theta > 0.f) || std::isinf(rope_theta)) return FC_ERR_ARG;
  PagedStoreArgs a;
  a.pool = view_of(pages, layer);
  a.table = table; a.width = table_width; a.kv_len = kv_len; a.qkv = qkv; a.qkv_stride = qkv_stride; a.q = q_out;
  a.c = c; a.hq = n_heads; a.hd = hd;
  rope_turns(rope_theta, hd, a.turns);
  const int units = (n_heads + 2 * pages->n_kv_heads) * (hd >> 3);
  const dim3 grid(batch * c, (units + 255) / 256);
  if (pages->dtype == FC_F32) paged_store_kernel<float><<<grid, 256, 0, (cudaStream_t)cuda_stream>>>(a);
  else paged_store_kernel<__nv_bfloat16><<<grid, 256, 0, (cudaStream_t)cuda_stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? FC_OK : FC_ERR_CUDA;
}

// The smallest size that is given out: such a call uses no scratch.
constexpr size_t kNoScratch = 256;

extern "C" size_t fc_op_paged_attention_scratch_bytes(int32_t batch, int32_t c, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                                      int32_t dtype, int32_t table_width, int32_t page_size, int32_t window, int32_t n_sink) {
  if (shape_ok(table_width, page_size, n_kv_heads, head_dim, batch, c, n_heads) || (dtype != FC_F32 && dtype != FC_BF16) || window < 0 || n_sink < 0) return 0;
  const PagedPlan plan = paged_plan(batch, c, n_heads, n_kv_heads, head_dim, dtype == FC_F32, table_width * page_size, window, window > 0 ? n_sink : 0);
  return !plan.fits ? 0 : plan.scratch == 0 ? kNoScratch : kNoScratch + (plan.scratch + 255) / 256 * 256;
}

extern "C" int fc_op_paged_attention(const fc_pages *pages, int32_t layer, const int32_t *table, int32_t table_width, const int32_t *kv_len,
                                     const void *q, int64_t q_stride, float *out, int32_t batch, int32_t c, int32_t n_heads,
                                     int32_t window, int32_t n_sink, void *scratch, size_t scratch_bytes, void *cuda_stream) {
  if (int rc = call_ok(pages, layer, table, table_width, kv_len, batch, c, n_heads)) return rc;
  const int hd = pages->head_dim, per = pages->dtype == FC_F32 ? 4 : 8;
  if (!q || !out || ((uintptr_t)q | (uintptr_t)out) % 16 || (uintptr_t)scratch % 256 || q_stride % per ||
      q_stride < (int64_t)n_heads * hd || window < 0 || n_sink < 0) return FC_ERR_ARG;
  PagedAttnArgs a; memset(&a, 0, sizeof a);
  a.pool = view_of(pages, layer);
  a.table = table; a.width = table_width; a.cap = table_width * pages->page_size; a.kv_len = kv_len; a.q = q; a.q_stride = q_stride; a.out = out;
  a.batch = batch; a.c = c; a.hq = n_heads; a.window = window; a.n_sink = window > 0 ? n_sink : 0; a.parts = (float *)scratch;
  const PagedPlan plan = paged_plan(batch, c, n_heads, pages->n_kv_heads, hd, pages->dtype == FC_F32, a.cap, window, a.n_sink);
  if (!plan.fits) return FC_ERR_CAPACITY;
  if (plan.scratch && !scratch) return FC_ERR_ARG;
  if (scratch_bytes < plan.scratch) return FC_ERR_CAPACITY;
  return launch_paged_attn(a, plan, pages->dtype, hd, (cudaStream_t)cuda_stream) == cudaSuccess ? FC_OK : FC_ERR_CUDA;
}
