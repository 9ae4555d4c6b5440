// New rows of block tables from old ones, and who holds which page (atspeed_op_fork_pages).
//   kept_j = ceil(len_j / page) entries of the parent's row; a partial last one: the parent's heir (the child with the largest
//   (len, -j)) goes on in it if its count is at most 1, the others copy it to the next free page
//   count' = count + handed out - old rows that hold the page + new rows that hold it;  free' = {page : count' <= 0}
// Bound: latency, for large tables HBM (the old entries in, the new ones out).
//
// One launch of clusters of eight CTAs.  Every CTA works out for itself which children are heirs and which page a copy gets (a few
// bytes a row, from L2, and one sum over the rows) instead of waiting for another launch.  The first cluster then makes the counts
// and the free list, in phases with the cluster's barrier between them; the other clusters write the rows.  An old row and the
// child that counts for it cancel: only the entries that a row gains or loses touch a count.
#include <algorithm>

#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kCluster = 8;
constexpr int kMaxPages = 1 << 26;

struct ForkArgs {
  int n_old, n_new, width, page, n_pages;
  const int *table, *kv_len, *q_len, *old_state, *parent, *length, *ref, *free, *n_free, *used;
  int *new_table, *new_len, *new_state, *src, *dst, *new_ref, *new_free, *new_n_free;
};

// What becomes of a new row.
struct Child {
  int parent, len, state;
  int kept;   // pages
};

__device__ __forceinline__ long long held_of(const ForkArgs& a, int p) {
  const long long kv = max(0, __ldg(a.kv_len + p));
  return kv + (a.q_len && (!a.old_state || __ldg(a.old_state + p) == ATSPEED_PLAN_OK) ? max(0, __ldg(a.q_len + p)) : 0);
}
__device__ __forceinline__ int pages_of(long long tokens, int page) { return (int)min((tokens + page - 1) / page, 0x7fffffffLL); }
__device__ __forceinline__ int held_pages(const ForkArgs& a, int p) { return min(a.width, pages_of(held_of(a, p), a.page)); }

__device__ __forceinline__ Child child_of(const ForkArgs& a, int j) {
  Child c = {a.parent ? __ldg(a.parent + j) : j, 0, ATSPEED_PLAN_OK, 0};
  if (c.parent < 0) return c;
  const long long held = c.parent < a.n_old ? held_of(a, c.parent) : -1;
  const long long len = a.length ? (long long)__ldg(a.length + j) : held;
  if (len < 0 || len > held || len > 0x7fffffff || pages_of(len, a.page) > a.width) {
    c.state = ATSPEED_PLAN_LIMIT;
    return c;
  }
  c.len = (int)len;
  c.kept = pages_of(len, a.page);
  return c;
}

constexpr int kNoCopy = -1, kNoPage = -2;   // in place of a copy's number

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads) fork_pages_kernel(const __grid_constant__ ForkArgs a) {
  extern __shared__ __align__(16) unsigned char raw[];
  unsigned long long* heir = reinterpret_cast<unsigned long long*>(raw);   // [n_old] (len, ~j) of its best child, 0: none
  int* copy = reinterpret_cast<int*>(heir + a.n_old);                     // [n_new] which of the copies it is
  __shared__ int s_sum[kWarps], s_count[kCluster];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster_ctarank();
  const auto scan = [&](int v, int& all) {   // the sum over the threads before this one
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) s_sum[warp] = x;
    __syncthreads();
    if (warp == 0) {
      int y = s_sum[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int z = __shfl_up_sync(0xffffffffu, y, o);
        if (lane >= o) y += z;
      }
      s_sum[lane] = y;
    }
    __syncthreads();
    all = s_sum[kWarps - 1];
    return x - v + (warp ? s_sum[warp - 1] : 0);
  };
  const auto in_pool = [&](int e) { return (unsigned)e < (unsigned)a.n_pages; };
  const int n_free = max(0, __ldg(a.n_free)), used = a.used ? min(n_free, max(0, __ldg(a.used))) : 0;

  for (int p = tid; p < a.n_old; p += kThreads) heir[p] = 0;
  __syncthreads();
  for (int j = tid; j < a.n_new; j += kThreads) {
    const Child c = child_of(a, j);
    if (c.parent >= 0 && c.state == ATSPEED_PLAN_OK)
      atomicMax(heir + c.parent, (unsigned long long)(uint32_t)c.len << 32 | (uint32_t)~j);
  }
  __syncthreads();
  const auto is_heir = [&](const Child& c, int j) {
    return heir[c.parent] == ((unsigned long long)(uint32_t)c.len << 32 | (uint32_t)~j);
  };
  const auto last_entry = [&](const Child& c) { return __ldg(a.table + (long long)c.parent * a.width + c.kept - 1); };
  const int per = (a.n_new + kThreads - 1) / kThreads, j0 = min(a.n_new, tid * per), j1 = min(a.n_new, j0 + per);
  int mine = 0;
  for (int j = j0; j < j1; ++j) {
    const Child c = child_of(a, j);
    bool copies = false;
    if (c.parent >= 0 && c.len % a.page) {
      const int e = last_entry(c);
      copies = in_pool(e) && !(is_heir(c, j) && __ldg(a.ref + e) <= 1);
    }
    copy[j] = copies ? 0 : kNoCopy;
    mine += copies;
  }
  int all;
  int nth = scan(mine, all);
  for (int j = j0; j < j1; ++j)
    if (copy[j] != kNoCopy) {
      copy[j] = nth < n_free - used ? nth : kNoPage;
      ++nth;
    }
  __syncthreads();
  const auto fresh_page = [&](int j) { return __ldg(a.free + used + copy[j]); };

  if (blockIdx.x >= kCluster) {   // rows, a warp each
    const int warps = (gridDim.x - kCluster) * kWarps;
    for (int j = (blockIdx.x - kCluster) * kWarps + warp; j < a.n_new; j += warps) {
      const Child c = child_of(a, j);
      const int k = copy[j];
      const bool served = c.state == ATSPEED_PLAN_OK && k != kNoPage;
      const int kept = served ? c.kept : 0, fresh = k >= 0 ? fresh_page(j) : -1;
      const int* from = a.table + (long long)max(0, c.parent) * a.width;
      int* to = a.new_table + (long long)j * a.width;
      for (int i = lane; i < a.width; i += 32) to[i] = i < kept ? (k >= 0 && i == kept - 1 ? fresh : __ldg(from + i)) : -1;
      if (lane == 0) {
        a.new_len[j] = served ? c.len : -1;
        a.new_state[j] = c.state != ATSPEED_PLAN_OK ? c.state : served ? ATSPEED_PLAN_OK : ATSPEED_PLAN_NO_PAGES;
        a.src[j] = k >= 0 ? last_entry(c) : -1;
        a.dst[j] = fresh;
      }
    }
    return;
  }
  // counts: the old ones, then what changes
  for (int p = rank * kThreads + tid; p < a.n_pages; p += kCluster * kThreads) a.new_ref[p] = __ldg(a.ref + p);
  cluster_sync();
  const auto add = [&](int e, int v) {
    if (in_pool(e)) atomicAdd(a.new_ref + e, v);
  };
  for (int i = rank * kThreads + tid; i < used; i += kCluster * kThreads) add(__ldg(a.free + i), 1);
  for (int j = rank * kWarps + warp; j < a.n_new; j += kCluster * kWarps) {
    const Child c = child_of(a, j);
    if (c.parent < 0 || c.state != ATSPEED_PLAN_OK || copy[j] == kNoPage) continue;
    const int* from = a.table + (long long)c.parent * a.width;
    const int kept = c.kept - (copy[j] >= 0);
    if (is_heir(c, j)) {   // (with its parent's own hold)
      for (int i = kept + lane, n = held_pages(a, c.parent); i < n; i += 32) add(__ldg(from + i), -1);
    } else {
      for (int i = lane; i < kept; i += 32) add(__ldg(from + i), 1);
    }
    if (lane == 0 && copy[j] >= 0) add(fresh_page(j), 1);
  }
  for (int p = rank * kWarps + warp; p < a.n_old; p += kCluster * kWarps) {
    if (heir[p] && copy[~(uint32_t)heir[p]] != kNoPage) continue;   // (its heir has counted for it)
    const int* from = a.table + (long long)p * a.width;
    for (int i = lane, n = held_pages(a, p); i < n; i += 32) add(__ldg(from + i), -1);
  }
  cluster_sync();
  // the free list: every CTA a range of pages, in order
  const int share = (int)((a.n_pages + (long long)kCluster * kThreads - 1) / (kCluster * kThreads)) * kThreads;
  const int p0 = (int)min((long long)a.n_pages, (long long)rank * share), p1 = min(a.n_pages, p0 + share);
  int zeros = 0;
  for (int p = p0 + tid; p < p1; p += kThreads) zeros += __ldcg(a.new_ref + p) <= 0;
  scan(zeros, all);
  if (tid < kCluster) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa_u32(&s_count[rank], tid)), "r"(all) : "memory");
  }
  cluster_sync();
  int at = 0, total = 0;
  for (int r = 0; r < kCluster; ++r) {
    at += r < rank ? s_count[r] : 0;
    total += s_count[r];
  }
  for (int p = p0; p < p1; p += kThreads) {
    const bool is_free = p + tid < p1 && __ldcg(a.new_ref + p + tid) <= 0;
    const int before = scan(is_free, all);
    if (is_free) a.new_free[at + before] = p + tid;
    at += all;
  }
  for (int i = total + rank * kThreads + tid; i < a.n_pages; i += kCluster * kThreads) a.new_free[i] = -1;
  if (rank == 0 && tid == 0) *a.new_n_free = total;
  cluster_sync();   // (no CTA leaves while others may write to its counts)
}

}  // namespace
}  // namespace atspeed

using namespace atspeed;

extern "C" atspeed_status atspeed_op_fork_pages(atspeed_stream stream, int n_old, int n_new, const int32_t* d_table, int table_width,
                                                int page_size, const int32_t* d_kv_len, const int32_t* d_q_len,
                                                const int32_t* d_old_state, const int32_t* d_parent, const int32_t* d_length,
                                                int n_pages, const int32_t* d_ref, const int32_t* d_free,
                                                const int32_t* d_n_free, const int32_t* d_used, int32_t* d_new_table,
                                                int32_t* d_new_len, int32_t* d_new_state, int32_t* d_src, int32_t* d_dst,
                                                int32_t* d_new_ref, int32_t* d_new_free, int32_t* d_new_n_free) {
  if (!d_table || !d_kv_len || !d_ref || !d_free || !d_n_free || !d_new_table || !d_new_len || !d_new_state || !d_src || !d_dst ||
      !d_new_ref || !d_new_free || !d_new_n_free || n_old <= 0 || n_new <= 0 || table_width <= 0 || page_size <= 0 || n_pages <= 0)
    return ATSPEED_E_ARG;
  if ((!d_parent && n_old != n_new) || d_new_table == d_table || d_new_ref == d_ref || d_new_free == d_free) return ATSPEED_E_ARG;
  if (n_old > kMaxRequests || n_new > kMaxRequests || n_pages > kMaxPages) return ATSPEED_E_SHAPE;
  const ForkArgs a = {n_old,  n_new,  table_width, page_size,   n_pages,   d_table,   d_kv_len, d_q_len, d_old_state, d_parent,  d_length,
                      d_ref,  d_free, d_n_free,    d_used,      d_new_table, d_new_len, d_new_state, d_src, d_dst, d_new_ref, d_new_free,
                      d_new_n_free};
  const int smem = n_old * (int)sizeof(unsigned long long) + n_new * (int)sizeof(int);
  static std::atomic<unsigned long long> done{0};
  if (smem_attr_once(done, fork_pages_kernel, kMaxRequests * 12) != cudaSuccess) return ATSPEED_E_CUDA;
  // one cluster for the counts, and of the others what fills the GPU where there are rows enough (a warp a row)
  const int clusters = 1 + std::min(17, (n_new + kCluster * kWarps - 1) / (kCluster * kWarps));
  fork_pages_kernel<<<clusters * kCluster, kThreads, smem, (cudaStream_t)stream>>>(a);
  return launch_status();
}
