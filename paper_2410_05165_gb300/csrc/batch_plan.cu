// Block tables and slot maps of a serving step, from the requests' lengths (atspeed_op_batch_plan).
//   have_b = ceil(kv_b / page), need_b = ceil((kv_b + q_b) / page), new_b = need_b - have_b
//   served: new_b = 0 or new_0 + .. + new_b <= free;  its pages are free[new_0 + .. + new_(b-1) ..]
//   token i of request b: position p = kv_b + i of the cache, slot = page(p / page) * page + p mod page
//   ancestors of node i: i, parent(i), parent(parent(i)), ..; its depth is their number - 1
// Bound: latency (a few hundred KB at most).  Every CTA works out the prefix sums of all requests for itself (8 bytes a
// request from L2) instead of waiting for another kernel or CTA, then takes a share of the tokens, table rows and masks.
// 16 requests of 240 tree tokens take 5.6 us, 1021 single tokens 7.2 (launch included, in a graph).
#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kThreads = 256;
constexpr int kMaskLaneWords = 4;   // words of a mask row a lane holds: 128 words, 4096 tokens of a request

struct PlanArgs {
  int n, page, width, T, words;
  const int *q_len, *kv_len, *parent, *free, *n_free;
  int *table, *cu_q, *ctx_len, *state, *pages, *req, *pos;
  long long* slot;
  uint32_t* mask;
};

// Pages of a served request's tokens (unsigned: the sum may pass 2^31).
__device__ __forceinline__ int pages_of(const PlanArgs& a, int tokens) {
  return (int)(((unsigned)tokens + (unsigned)a.page - 1u) / (unsigned)a.page);
}

// Inclusive sums over the CTA's threads of two values each.
__device__ __forceinline__ void block_scan2(long long& a, long long& b, long long (*red)[2]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
    if (lane >= o) a += x, b += y;
  }
  if (lane == 31) red[warp][0] = a, red[warp][1] = b;
  __syncthreads();
  for (int w = 0; w < warp; ++w) a += red[w][0], b += red[w][1];
}

// start[b]: first token of request b;  base[b]: first of its new pages in the free list, -1: not served
__global__ void __launch_bounds__(kThreads) batch_plan_kernel(PlanArgs a) {
  extern __shared__ int sm[];
  __shared__ long long red[kThreads / 32][2];
  __shared__ int s_pages[2];   // taken, asked for up to the last served request
  int* start = sm;
  int* base = sm + a.n + 1;
  const int tid = threadIdx.x, per = (a.n + kThreads - 1) / kThreads;
  const int b0 = min(a.n, tid * per), b1 = min(a.n, b0 + per);
  const long long n_free = max(0, *a.n_free);
  if (tid < 2) s_pages[tid] = 0;
  // this thread's requests: tokens and new pages (a request past a limit takes neither pages nor, with a
  // negative length, tokens)
  auto request = [&](int b, long long first, long long& q, long long& fresh) {
    const long long ql = a.q_len[b], kv = a.kv_len[b];
    q = max(0LL, ql);
    const long long need = (kv + q + a.page - 1) / a.page;
    const bool ok = ql >= 0 && kv >= 0 && kv + q <= 0x7fffffff && need <= a.width && first + q <= a.T &&
                    (!a.mask || q <= 32LL * a.words);
    fresh = ok ? need - (kv + a.page - 1) / a.page : 0;
    return ok;
  };
  // (tokens first: whether a request's fit under max_tokens decides whether it takes pages)
  long long q_sum = 0, zero = 0;
  for (int b = b0; b < b1; ++b) q_sum += max(0, a.q_len[b]);
  const long long q_own = q_sum;
  block_scan2(q_sum, zero, red);
  __syncthreads();
  long long first = q_sum - q_own, f_sum = 0, q, fresh;
  long long at = first;
  for (int b = b0; b < b1; ++b) {
    request(b, at, q, fresh);
    at += q;
    f_sum += fresh;
  }
  const long long f_own = f_sum;
  zero = 0;
  block_scan2(f_sum, zero, red);
  long long upto = f_sum - f_own, took = 0, asked = 0;
  at = first;
  for (int b = b0; b < b1; ++b) {
    const bool ok = request(b, at, q, fresh);
    const bool served = ok && (fresh == 0 || upto + fresh <= n_free);
    start[b] = (int)min((long long)a.T, at);
    base[b] = served ? (int)min(upto, n_free) : -1;
    at += q;
    upto += fresh;
    if (served) asked = upto;
    if (served && fresh) took = upto;
    if (blockIdx.x == 0) {
      a.cu_q[b] = start[b];
      a.ctx_len[b] = served ? a.kv_len[b] : -1;
      a.state[b] = served ? ATSPEED_PLAN_OK : ok ? ATSPEED_PLAN_NO_PAGES : ATSPEED_PLAN_LIMIT;
    }
  }
  if (b1 == a.n && b0 < b1) {
    start[a.n] = (int)min((long long)a.T, at);
    if (blockIdx.x == 0) a.cu_q[a.n] = start[a.n];
  }
  if (took) atomicMax(&s_pages[0], (int)took);
  if (asked) atomicMax(&s_pages[1], (int)min(asked, 0x7fffffffLL));
  __syncthreads();
  if (blockIdx.x == 0 && tid < 2) a.pages[tid] = s_pages[tid];

  // table entries of the new pages, a thread a request
  for (int b = blockIdx.x * kThreads + tid; b < a.n; b += gridDim.x * kThreads) {
    if (base[b] < 0) continue;
    const int kv = a.kv_len[b], have = pages_of(a, kv), need = pages_of(a, kv + a.q_len[b]);
    for (int j = have; j < need; ++j) a.table[(size_t)b * a.width + j] = a.free[base[b] + j - have];
  }
  // tokens
  const int total = start[a.n];
  const auto find = [&](int t) {   // the last request whose first token is not past t
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (start[mid] <= t) lo = mid;
      else hi = mid - 1;
    }
    return lo;
  };
  const auto place = [&](int t, int b, int depth) {
    const int i = t - start[b], kv = a.kv_len[b];
    long long slot = -1;
    if (base[b] >= 0) {
      const int p = kv + i, col = p / a.page, have = pages_of(a, kv);
      const int id = col < have ? a.table[(size_t)b * a.width + col] : a.free[base[b] + col - have];
      slot = (long long)id * a.page + p % a.page;
    }
    a.req[t] = b;
    a.pos[t] = (int)((unsigned)kv + depth);
    a.slot[t] = slot;
  };
  if (!a.mask) {
    for (int t = blockIdx.x * kThreads + tid; t < a.T; t += gridDim.x * kThreads) {
      if (t < total) {
        const int b = find(t);
        place(t, b, t - start[b]);
      } else {
        a.req[t] = -1;
        a.pos[t] = 0;
        a.slot[t] = -1;
      }
    }
    return;
  }
  // trees, a warp a token: the walk up in every lane, each keeping its words of the row
  const int lane = tid & 31;
  for (int t = blockIdx.x * (kThreads / 32) + (tid >> 5); t < a.T; t += gridDim.x * (kThreads / 32)) {
    uint32_t w[kMaskLaneWords] = {};
    if (t < total) {
      const int b = find(t), first_t = start[b], len = min(start[b + 1] - first_t, 32 * a.words);
      int node = t - first_t, depth = -1;
      for (int step = 0; step < len && node >= 0 && node < len; ++step) {   // (a cycle ends after len steps)
        ++depth;
#pragma unroll
        for (int k = 0; k < kMaskLaneWords; ++k)
          if ((node >> 5) == lane + 32 * k) w[k] |= 1u << (node & 31);
        node = __ldg(a.parent + first_t + node);
      }
      if (lane == 0) place(t, b, max(0, depth));
    } else if (lane == 0) {
      a.req[t] = -1;
      a.pos[t] = 0;
      a.slot[t] = -1;
    }
#pragma unroll
    for (int k = 0; k < kMaskLaneWords; ++k)
      if (lane + 32 * k < a.words) a.mask[(size_t)t * a.words + lane + 32 * k] = w[k];
  }
}

}  // namespace
}  // namespace atspeed

using namespace atspeed;

extern "C" atspeed_status atspeed_op_batch_plan(atspeed_stream stream, int n_req, const int32_t* d_q_len,
                                                const int32_t* d_kv_len, const int32_t* d_parent, int page_size,
                                                int32_t* d_block_table, int table_width, const int32_t* d_free,
                                                const int32_t* d_n_free, int max_tokens, int mask_words, int32_t* d_cu_q,
                                                int32_t* d_ctx_len, int32_t* d_state, int32_t* d_pages, int32_t* d_req,
                                                int32_t* d_pos, int64_t* d_slot, uint32_t* d_mask) {
  if (!d_q_len || !d_kv_len || !d_block_table || !d_free || !d_n_free || !d_cu_q || !d_ctx_len || !d_state || !d_pages ||
      !d_req || !d_pos || !d_slot || n_req <= 0 || page_size <= 0 || table_width <= 0 || max_tokens <= 0)
    return ATSPEED_E_ARG;
  if ((d_parent != nullptr) != (d_mask != nullptr) || (d_mask && mask_words <= 0)) return ATSPEED_E_ARG;
  if (n_req > kMaxRequests || (d_mask && mask_words > 32 * kMaskLaneWords)) return ATSPEED_E_SHAPE;
  const PlanArgs a = {n_req,  page_size,     table_width, max_tokens, d_mask ? mask_words : 0, d_q_len, d_kv_len, d_parent,
                      d_free, d_n_free,      d_block_table, d_cu_q,   d_ctx_len, d_state,      d_pages, d_req,    d_pos,
                      reinterpret_cast<long long*>(d_slot), d_mask};
  const int smem = (2 * n_req + 1) * (int)sizeof(int);
  static std::atomic<unsigned long long> done{0};
  if (smem_attr_once(done, batch_plan_kernel, (2 * kMaxRequests + 1) * (int)sizeof(int)) != cudaSuccess)
    return ATSPEED_E_CUDA;
  const long long items = d_mask ? max_tokens : (max_tokens + 31LL) / 32, most = 304;
  const long long want = max((items + kThreads / 32 - 1) / (kThreads / 32), (n_req + kThreads - 1LL) / kThreads);
  batch_plan_kernel<<<(int)(want < most ? want : most), kThreads, smem, (cudaStream_t)stream>>>(a);
  return launch_status();
}
