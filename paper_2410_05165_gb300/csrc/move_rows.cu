// Rows of paged caches that change their place, in all layers at once: the filled part of pages to other pages
// (atspeed_op_copy_pages) and an accepted path's tokens behind the cached ones (atspeed_op_compact_tokens).
// Bound: HBM (each moved byte read once and written once); few bytes: the launch and the chain lengths -> rows.
#include <algorithm>

#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kLayers = 120;   // of a launch (their addresses are kernel parameters: 4 KB)
constexpr int kBatch = 8;      // 16-byte loads that a thread has under way

struct Geometry {   // the same in all layers, in 16-byte vectors
  int n_pages, page, heads, vecs;   // vecs: of a head's row
  long long k_page, k_token, k_head, v_page, v_token, v_head;
};
struct Layers {
  uint4* at[kLayers][2];   // K, V
};

struct CopyArgs {
  Geometry g;
  int layers, n;
  const int *src, *dst, *length;
  Layers l;
};

struct CompactArgs {
  Geometry g;
  int layers, n, T, keep_width;
  const long long* slot;
  const int *cu_q, *kv_len, *state, *keep, *n_keep;
  int* new_len;   // null: not of this launch
  Layers l;
};

// A CTA takes (copy, layer, K or V) after (copy, layer, K or V).
__global__ void __launch_bounds__(kThreads) copy_pages_kernel(const __grid_constant__ CopyArgs a) {
  const Geometry& g = a.g;
  const long long items = 2LL * a.n * a.layers;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int j = (int)(it / (2 * a.layers)), lv = (int)(it % (2 * a.layers));
    const int src = __ldg(a.src + j), dst = __ldg(a.dst + j);
    if ((unsigned)src >= (unsigned)g.n_pages || (unsigned)dst >= (unsigned)g.n_pages || src == dst) continue;
    const int len = a.length ? __ldg(a.length + j) : g.page;
    if (len < 1) continue;
    const int rows = (len - 1) % g.page + 1;
    const bool v = lv & 1;
    uint4* base = a.l.at[lv >> 1][lv & 1];
    const long long sp = v ? g.v_page : g.k_page, st = v ? g.v_token : g.k_token, sh = v ? g.v_head : g.k_head;
    const int row = g.heads * g.vecs;
    const long long all = (long long)rows * row;
    for (long long i = threadIdx.x; i < all; i += kThreads) {
      const int t = (int)(i / row), h = (int)(i % row) / g.vecs, c = (int)(i % row) % g.vecs;
      const long long at = t * st + h * sh + c;
      base[dst * sp + at] = base[src * sp + at];
    }
  }
}

// The moves of a request: a thread has 16 bytes of a row, in one layer's K or V, and moves them for token after token, so that a
// row is read before a later move of the same bytes writes to it (a kept token's place is never behind its own).
__global__ void __launch_bounds__(kThreads) compact_tokens_kernel(const __grid_constant__ CompactArgs a) {
  const Geometry& g = a.g;
  const int b = blockIdx.x, lv = blockIdx.y, tid = threadIdx.x;
  const int q0 = min(a.T, max(0, __ldg(a.cu_q + b))), q = min(a.T, __ldg(a.cu_q + b + 1)) - q0;
  int n = !a.state || __ldg(a.state + b) == ATSPEED_PLAN_OK ? min(a.keep_width, __ldg(a.n_keep + b)) : 0;
  const int* keep = a.keep + (long long)b * a.keep_width;
  int count = 0;   // of the list up to its first entry that is out of order
  for (int last = -1; count < n; ++count) {
    const int k = __ldg(keep + count);
    if (k <= last || k >= q) break;
    last = k;
  }
  if (a.new_len && lv == 0 && blockIdx.z == 0 && tid == 0) a.new_len[b] = __ldg(a.kv_len + b) + count;
  const bool v = lv & 1;
  uint4* base = a.l.at[lv >> 1][lv & 1];
  const long long sp = v ? g.v_page : g.k_page, st = v ? g.v_token : g.k_token, sh = v ? g.v_head : g.k_head;
  const long long rows = (long long)g.n_pages * g.page;
  for (int i = blockIdx.z * kThreads + tid; i < g.heads * g.vecs; i += gridDim.z * kThreads) {
    uint4* at = base + i / g.vecs * sh + i % g.vecs;
    for (int m = 0; m < count; ++m) {
      const int k = __ldg(keep + m);
      if (k == m) continue;
      const long long from = __ldg(a.slot + q0 + k), to = __ldg(a.slot + q0 + m);
      if ((unsigned long long)from >= (unsigned long long)rows || (unsigned long long)to >= (unsigned long long)rows) continue;
      at[to / g.page * sp + to % g.page * st] = at[from / g.page * sp + from % g.page * st];
    }
  }
}

// Checks layers of one geometry.
atspeed_status geometry_of(const atspeed_kv_pages* l, int n, Geometry& g) {
  if (!l || n <= 0) return ATSPEED_E_ARG;
  for (int i = 0; i < n; ++i) {
    if (const atspeed_status s = check_pages(l + i)) return s;
    const bool same = l[i].k_type == l[0].k_type && l[i].v_type == l[0].v_type && l[i].n_pages == l[0].n_pages &&
                      l[i].page_size == l[0].page_size && l[i].n_kv_heads == l[0].n_kv_heads && l[i].head_dim == l[0].head_dim &&
                      std::equal(l[i].k_stride, l[i].k_stride + 3, l[0].k_stride) &&
                      std::equal(l[i].v_stride, l[i].v_stride + 3, l[0].v_stride);
    if (!same) return ATSPEED_E_ARG;
  }
  if (l->head_dim % 8 || (long long)l->n_kv_heads * l->head_dim > 1 << 24 || l->page_size > 1 << 20) return ATSPEED_E_SHAPE;
  g = {l->n_pages,         l->page_size,       l->n_kv_heads,      l->head_dim / 8,     l->k_stride[0] / 8,
       l->k_stride[1] / 8, l->k_stride[2] / 8, l->v_stride[0] / 8, l->v_stride[1] / 8, l->v_stride[2] / 8};
  return ATSPEED_OK;
}

int set_layers(Layers& to, const atspeed_kv_pages* l, int first, int n) {
  const int m = std::min(kLayers, n - first);
  for (int i = 0; i < m; ++i) to.at[i][0] = static_cast<uint4*>(l[first + i].d_k), to.at[i][1] = static_cast<uint4*>(l[first + i].d_v);
  return m;
}

}  // namespace
}  // namespace atspeed

using namespace atspeed;

extern "C" atspeed_status atspeed_op_copy_pages(atspeed_stream stream, const atspeed_kv_pages* layers, int n_layers, int n,
                                                const int32_t* d_src, const int32_t* d_dst, const int32_t* d_length) {
  if (!d_src || !d_dst || n <= 0) return ATSPEED_E_ARG;
  CopyArgs a = {};
  if (const atspeed_status s = geometry_of(layers, n_layers, a.g)) return s;
  a.n = n, a.src = d_src, a.dst = d_dst, a.length = d_length;
  for (int first = 0; first < n_layers; first += kLayers) {
    a.layers = set_layers(a.l, layers, first, n_layers);
    const int grid = (int)std::min(152LL * 8, 2LL * n * a.layers);
    copy_pages_kernel<<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
  }
  return launch_status();
}

extern "C" atspeed_status atspeed_op_compact_tokens(atspeed_stream stream, const atspeed_kv_pages* layers, int n_layers, int n_req,
                                                    int T, const int64_t* d_slot, const int32_t* d_cu_q, const int32_t* d_kv_len,
                                                    const int32_t* d_state, const int32_t* d_keep, int keep_width,
                                                    const int32_t* d_n_keep, int32_t* d_new_len) {
  if (!d_slot || !d_cu_q || !d_kv_len || !d_keep || !d_n_keep || !d_new_len || n_req <= 0 || T <= 0 || keep_width <= 0)
    return ATSPEED_E_ARG;
  CompactArgs a = {};
  if (const atspeed_status s = geometry_of(layers, n_layers, a.g)) return s;
  if (n_req > kMaxRequests) return ATSPEED_E_SHAPE;
  a.n = n_req, a.T = T, a.keep_width = keep_width, a.slot = reinterpret_cast<const long long*>(d_slot), a.cu_q = d_cu_q;
  a.kv_len = d_kv_len, a.state = d_state, a.keep = d_keep, a.n_keep = d_n_keep;
  for (int first = 0; first < n_layers; first += kLayers) {
    a.layers = set_layers(a.l, layers, first, n_layers);
    a.new_len = first == 0 ? d_new_len : nullptr;
    const dim3 grid(n_req, 2 * a.layers, std::min(64, (a.g.heads * a.g.vecs + kThreads - 1) / kThreads));
    compact_tokens_kernel<<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
  }
  return launch_status();
}
