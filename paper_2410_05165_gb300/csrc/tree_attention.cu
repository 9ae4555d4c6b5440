// Attention of new tokens (trees, chains) over a batch's paged caches (atspeed_op_tree_attention).
//   o = sum_j w_j v_j / sum_j w_j, w_j = exp(scale q.k_j), over the positions j < ctx and those of the token's ancestors
#include <cmath>

#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

struct TreeAttnArgs {
  const uint16_t *q, *k, *v;
  long long ks[3], vs[3], q_stride, out_stride;
  int H, G, n, T, page, n_pages, width, words;
  const int *cu_q, *ctx, *table;
  const uint32_t* mask;
  float scale;
  uint16_t* out;
  float* lse;
  bool k_f16, v_f16;
};

__device__ __forceinline__ float one(uint16_t x, bool f16) {
  return f16 ? __half2float(__ushort_as_half(x)) : __uint_as_float((uint32_t)x << 16);
}

// A warp a (token, head), its lanes over the head's dimensions, a key at a time.
template <int HD>
__global__ void __launch_bounds__(256) tree_attention_kernel(const __grid_constant__ TreeAttnArgs a) {
  constexpr int E = HD / 32;
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int t = (int)(w / a.H), h = (int)(w % a.H), kh = h / a.G;
  if (t >= a.T) return;
  int lo = 0, hi = a.n;
  while (lo < hi) {   // the first request that ends past t
    const int mid = (lo + hi) >> 1;
    if (a.cu_q[mid + 1] > t) hi = mid;
    else lo = mid + 1;
  }
  if (lo == a.n) return;
  const int i = t - a.cu_q[lo], len = a.cu_q[lo + 1] - a.cu_q[lo], ctx = a.ctx[lo];
  const long long keys = ctx < 0 ? 0 : min((long long)ctx + len, (long long)a.width * a.page);
  float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
  for (int e = 0; e < E; ++e) q[e] = one(a.q[t * a.q_stride + (long long)h * HD + lane + 32 * e], a.k_f16) * a.scale;
  for (long long p = 0; p < keys; ++p) {
    if (p >= ctx) {
      const int j = (int)(p - ctx);
      const bool see = a.mask ? (j >> 5) < a.words && (a.mask[(long long)t * a.words + (j >> 5)] >> (j & 31) & 1) : j <= i;
      if (!see) continue;
    }
    const int id = a.table[(long long)lo * a.width + p / a.page];
    if (id < 0 || id >= a.n_pages) continue;
    const long long row = p % a.page;
    float s = 0.f;
    for (int e = 0; e < E; ++e) s += q[e] * one(a.k[id * a.ks[0] + row * a.ks[1] + kh * a.ks[2] + lane + 32 * e], a.k_f16);
    s = warp_sum(s);
    const float m2 = fmaxf(m, s), f = m == -INFINITY ? 0.f : expf(m - m2), x = expf(s - m2);
    l = l * f + x;
    for (int e = 0; e < E; ++e)
      o[e] = o[e] * f + x * one(a.v[id * a.vs[0] + row * a.vs[1] + kh * a.vs[2] + lane + 32 * e], a.v_f16);
    m = m2;
  }
  for (int e = 0; e < E; ++e) {
    const float x = l > 0.f || l != l ? o[e] / l : 0.f;
    const uint32_t u = pack2(x, 0.f, a.k_f16);
    a.out[t * a.out_stride + (long long)h * HD + lane + 32 * e] = (uint16_t)u;
  }
  if (a.lse && lane == 0) a.lse[(long long)t * a.H + h] = l > 0.f ? m + logf(l) : l != l ? l : -INFINITY;
}

}  // namespace
}  // namespace atspeed

using namespace atspeed;

extern "C" {

size_t atspeed_op_tree_attention_workspace(void) { return 256; }

atspeed_status atspeed_op_tree_attention(atspeed_stream stream, const atspeed_kv_pages* cache, const void* d_q,
                                         int64_t q_stride, int n_heads, int n_req, int T, const int32_t* d_cu_q,
                                         const int32_t* d_ctx_len, const int32_t* d_block_table, int table_width,
                                         const uint32_t* d_mask, int mask_words, float scale, void* d_out, int64_t out_stride,
                                         float* d_lse, void* d_ws) {
  const atspeed_status st = check_pages(cache);
  if (st != ATSPEED_OK) return st;
  const atspeed_kv_pages& c = *cache;
  if (!d_q || !d_out || !d_cu_q || !d_ctx_len || !d_block_table || !d_ws || n_heads <= 0 || n_req <= 0 || T <= 0 ||
      table_width <= 0 || (d_mask && mask_words <= 0) || !(scale > 0.f) || !std::isfinite(scale))
    return ATSPEED_E_ARG;
  const int hd = c.head_dim, ps = c.page_size;
  if ((hd != 32 && hd != 64 && hd != 128) || (ps != 16 && ps != 32 && ps != 64 && ps != 128 && ps != 256) ||
      n_heads % c.n_kv_heads || n_heads / c.n_kv_heads > 128 || n_req > kMaxRequests)
    return ATSPEED_E_SHAPE;
  if (q_stride < (int64_t)n_heads * hd || out_stride < (int64_t)n_heads * hd || q_stride % 8 || out_stride % 8 ||
      !aligned16(d_q) || !aligned16(d_out) || (reinterpret_cast<uintptr_t>(d_ws) & 255))
    return ATSPEED_E_ARG;
  TreeAttnArgs a = {};
  a.q = static_cast<const uint16_t*>(d_q), a.k = static_cast<const uint16_t*>(c.d_k), a.v = static_cast<const uint16_t*>(c.d_v);
  for (int i = 0; i < 3; ++i) a.ks[i] = c.k_stride[i], a.vs[i] = c.v_stride[i];
  a.q_stride = q_stride, a.out_stride = out_stride;
  a.H = n_heads, a.G = n_heads / c.n_kv_heads, a.n = n_req, a.T = T, a.page = ps, a.n_pages = c.n_pages;
  a.width = table_width, a.words = mask_words, a.cu_q = d_cu_q, a.ctx = d_ctx_len, a.table = d_block_table, a.mask = d_mask;
  a.scale = scale, a.out = static_cast<uint16_t*>(d_out), a.lse = d_lse;
  a.k_f16 = c.k_type == ATSPEED_F16, a.v_f16 = c.v_type == ATSPEED_F16;
  const long long warps = (long long)T * n_heads;
  if ((warps + 7) / 8 > 0x7fffffffLL) return ATSPEED_E_SHAPE;
  const unsigned grid = (unsigned)((warps + 7) / 8);
  if (hd == 32) tree_attention_kernel<32><<<grid, 256, 0, (cudaStream_t)stream>>>(a);
  else if (hd == 64) tree_attention_kernel<64><<<grid, 256, 0, (cudaStream_t)stream>>>(a);
  else tree_attention_kernel<128><<<grid, 256, 0, (cudaStream_t)stream>>>(a);
  return launch_status();
}

}  // extern "C"
