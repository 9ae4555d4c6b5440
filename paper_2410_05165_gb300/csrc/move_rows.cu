// Rows of paged caches that change their place, in all layers at once: the filled part of pages to other pages
// (atspeed_op_copy_pages) and an accepted path's tokens behind the cached ones (atspeed_op_compact_tokens).
// Bound: HBM (each moved byte read once and written once); few bytes: the launch and the chain lengths -> rows.  Copies of 569 MB take
// 73 us, 7.8 TB/s (some of the writes stay in L2), of 1 MB 4.3.
#include <algorithm>

#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kLayers = 120;   // of a launch (their addresses are kernel parameters: 4 KB)
constexpr int kBatch = 6;      // 16-byte loads that a thread has under way

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

// Copies from `from` to `to` what a warp has of one layer's K or V: i-th vectors at at(i), i < n, six under way a lane.
template <class At>
__device__ __forceinline__ void warp_copy(uint4* to, const uint4* from, int n, At&& at) {
  const int lane = threadIdx.x & 31;
  for (int i0 = lane; i0 < n; i0 += 32 * kBatch) {
    uint4 x[kBatch];
    long long o[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (i0 + 32 * q < n) {
        o[q] = at(i0 + 32 * q);
        x[q] = from[o[q]];
      }
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (i0 + 32 * q < n) to[o[q]] = x[q];
  }
}

// A warp takes some rows (512 vectors, a row at least) of a copy in one layer's K or V after some rows.  Copies come and go with the lengths,
// so every CTA lists 1024 of them at a time with the rows that they have, and the grid's warps share those out: with a CTA a (copy,
// layer, K or V) and pairs of -1 among them, the 569 MB took 118 us.  (344 pairs in two lists of 256: 18 us, in one 13.  Three or four CTAs an
// SM: the same for many bytes, 1 to 2 us more for few.)
constexpr int kPairs = 1024, kEach = kPairs / kThreads, kCopyCtas = 2;   // CTAs an SM
__global__ void __launch_bounds__(kThreads, kCopyCtas) copy_pages_kernel(const __grid_constant__ CopyArgs a) {
  __shared__ int s_upto[kPairs], s_src[kPairs], s_dst[kPairs], s_rows[kPairs], s_warp[kWarps];
  const Geometry& g = a.g;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, all_warps = gridDim.x * kWarps;
  const int row = g.heads * g.vecs, some = max(1, 512 / row);   // vectors of a row, rows that a warp takes at once
  long long turn = blockIdx.x * kWarps + warp;                  // this warp's next piece of work
  for (int j0 = 0; j0 < a.n; j0 += kPairs) {
    int src[kEach], dst[kEach], rows[kEach], upto = 0;
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      const int j = j0 + q * kThreads + tid;   // (the list's order does not matter)
      src[q] = dst[q] = -1, rows[q] = 0;
      if (j >= a.n) continue;
      src[q] = __ldg(a.src + j), dst[q] = __ldg(a.dst + j);
      const int len = a.length ? __ldg(a.length + j) : g.page;
      if ((unsigned)src[q] < (unsigned)g.n_pages && (unsigned)dst[q] < (unsigned)g.n_pages && src[q] != dst[q] && len > 0)
        rows[q] = (len - 1) % g.page + 1;
    }
#pragma unroll
    for (int q = 0; q < kEach; ++q) upto += (rows[q] + some - 1) / some;
    const int mine = upto;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    __syncthreads();   // (the list before this one is done with)
    if (lane == 31) s_warp[warp] = upto;
    __syncthreads();
    upto -= mine;
    for (int w = 0; w < warp; ++w) upto += s_warp[w];
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      upto += (rows[q] + some - 1) / some;
      const int at = tid * kEach + q;
      s_upto[at] = upto, s_src[at] = src[q], s_dst[at] = dst[q], s_rows[at] = rows[q];
    }
    __syncthreads();
    const int units = s_upto[kPairs - 1];
    const long long work = (long long)units * 2 * a.layers;
    for (; turn < work; turn += all_warps) {
      const int lv = (int)(turn / units), u = (int)(turn % units);
      int c = 0;   // the first copy whose work ends behind u
#pragma unroll
      for (int step = kPairs / 2; step > 0; step >>= 1)
        if (s_upto[c + step - 1] <= u) c += step;
      const int t0 = (u - (c ? s_upto[c - 1] : 0)) * some, n = min(some, s_rows[c] - t0);
      const bool v = lv & 1;
      uint4* base = a.l.at[lv >> 1][lv & 1];
      const long long sp = v ? g.v_page : g.k_page, st = v ? g.v_token : g.k_token, sh = v ? g.v_head : g.k_head;
      uint4* to = base + s_dst[c] * sp + t0 * st;
      const uint4* from = base + s_src[c] * sp + t0 * st;
      if (sh == g.vecs && (n == 1 || st == row)) {
        warp_copy(to, from, n * row, [](int i) { return (long long)i; });
      } else {
        warp_copy(to, from, n * row, [&](int i) {
          const int t = i / row, r = i - t * row, h = r / g.vecs;
          return t * st + h * sh + (r - h * g.vecs);
        });
      }
    }
    turn -= work;   // (the next list's first work goes to those that have none of this one's)
  }
}

// The moves of a request: a thread has 16 bytes of a row, in one layer's K or V, and moves them for token after token, so that a
// row is read before a later move of the same bytes writes to it (a kept token's place is never behind its own).  A CTA has two of
// them a thread, of as many layers as that takes (a CTA a layer's K or V: 63 us for 536 requests of 28 layers of one head).
// us: one path of three in 4 layers of 12 heads of 64 2.9, 16 paths in 32 layers of 32 heads of 128 (22 MB) 6.4.
constexpr int kMoves = 64;   // that the CTA works out at a time
__global__ void __launch_bounds__(kThreads) compact_tokens_kernel(const __grid_constant__ CompactArgs a) {
  __shared__ int s_count;
  __shared__ long long s_from[2][kMoves], s_to[2][kMoves];   // in K and in V: vectors from the base, to: -1 if it does not move
  const Geometry& g = a.g;
  const int b = blockIdx.x, tid = threadIdx.x, row = g.heads * g.vecs;
  const int q0 = min(a.T, max(0, __ldg(a.cu_q + b))), q = min(a.T, __ldg(a.cu_q + b + 1)) - q0;
  const int n = !a.state || __ldg(a.state + b) == ATSPEED_PLAN_OK ? max(0, min(a.keep_width, __ldg(a.n_keep + b))) : 0;
  const int* keep = a.keep + (long long)b * a.keep_width;
  if (tid == 0) s_count = n;
  __syncthreads();
  for (int i = tid; i < n; i += kThreads) {   // the list ends at its first entry that is out of order
    const int k = __ldg(keep + i), before = i ? __ldg(keep + i - 1) : -1;
    if (k <= before || k >= q) atomicMin(&s_count, i);
  }
  __syncthreads();
  const int count = s_count;
  if (a.new_len && blockIdx.y == 0 && tid == 0) a.new_len[b] = __ldg(a.kv_len + b) + count;
  const unsigned long long rows = (unsigned long long)g.n_pages * g.page;
  const int all = 2 * a.layers * row;   // vectors of a token
  for (int m0 = 0; m0 < count; m0 += kMoves) {
    if (m0) __syncthreads();
    if (tid < kMoves && m0 + tid < count) {
      const int k = __ldg(keep + m0 + tid);
      const unsigned long long from = (unsigned long long)__ldg(a.slot + q0 + k), to = (unsigned long long)__ldg(a.slot + q0 + m0 + tid);
      const bool moves = k != m0 + tid && from < rows && to < rows;   // (negative slots are large ones)
      const auto page_of = [&](unsigned long long r) { return r >> 32 ? r / g.page : (unsigned)r / (unsigned)g.page; };
      const long long p = (long long)page_of(from), q = (long long)page_of(to);
      const long long pr = (long long)from - p * g.page, qr = (long long)to - q * g.page;
      s_from[0][tid] = p * g.k_page + pr * g.k_token, s_from[1][tid] = p * g.v_page + pr * g.v_token;
      s_to[0][tid] = moves ? q * g.k_page + qr * g.k_token : -1, s_to[1][tid] = moves ? q * g.v_page + qr * g.v_token : -1;
    }
    __syncthreads();
    const int moves = min(kMoves, count - m0);
    for (int i = blockIdx.y * kThreads + tid; i < all; i += gridDim.y * kThreads) {
      const int lv = i / row, r = i - lv * row, h = r / g.vecs, v = lv & 1;
      uint4* at = a.l.at[lv >> 1][v] + h * (v ? g.v_head : g.k_head) + (r - h * g.vecs);
      // (four reads, then as many writes: those go to places before any later token's)
      for (int t = 0; t < moves; t += 4) {
        uint4 x[4];
        long long to[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          to[j] = t + j < moves ? s_to[v][t + j] : -1;
          if (to[j] >= 0) x[j] = at[s_from[v][t + j]];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (to[j] >= 0) at[to[j]] = x[j];
      }
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
  if (n > 0x7fffffff - kPairs) return ATSPEED_E_SHAPE;   // (a list past the last pair begins below 2^31)
  a.n = n, a.src = d_src, a.dst = d_dst, a.length = d_length;
  for (int first = 0; first < n_layers; first += kLayers) {
    a.layers = set_layers(a.l, layers, first, n_layers);
    // (what runs at once; few copies: a warp a row at most)
    const int grid = (int)std::min(152LL * kCopyCtas, (2LL * n * a.layers * std::min(64, a.g.page) + kWarps - 1) / kWarps);
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
  if (n_req > kMaxRequests || keep_width > 0x7fffffff - kThreads) return ATSPEED_E_SHAPE;   // (indices past the last entry stay below 2^31)
  // (a request's kept tokens are read by other CTAs than the one that writes its new length)
  const Span in[] = {{d_slot, 8ll * T}, {d_cu_q, 4ll * n_req + 4}, {d_kv_len == d_new_len ? nullptr : d_kv_len, 4ll * n_req}, {d_state, 4ll * n_req},
                     {d_keep, 4ll * n_req * keep_width}, {d_n_keep, 4ll * n_req}};
  const Span out[] = {{d_new_len, 4ll * n_req}};
  if (outputs_overlap(out, in)) return ATSPEED_E_ARG;
  a.n = n_req, a.T = T, a.keep_width = keep_width, a.slot = reinterpret_cast<const long long*>(d_slot), a.cu_q = d_cu_q;
  a.kv_len = d_kv_len, a.state = d_state, a.keep = d_keep, a.n_keep = d_n_keep;
  for (int first = 0; first < n_layers; first += kLayers) {
    a.layers = set_layers(a.l, layers, first, n_layers);
    a.new_len = first == 0 ? d_new_len : nullptr;
    const long long vectors = 2LL * a.layers * a.g.heads * a.g.vecs;
    const dim3 grid(n_req, (unsigned)std::min(65535LL, (vectors + 2 * kThreads - 1) / (2 * kThreads)));
    compact_tokens_kernel<<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
  }
  return launch_status();
}
