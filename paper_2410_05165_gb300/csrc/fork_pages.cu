// New rows of block tables from old ones, and who holds which page (atspeed_op_fork_pages).
//   kept_j = ceil(len_j / page) entries of the parent's row; a partial last one: the parent's heir (the child with the largest
//   (len, -j)) goes on in it if its count is at most 1, the others copy it to the next free page
//   count' = count + handed out - old rows that hold the page + new rows that hold it;  free' = {page : count' <= 0}
// Bound: latency, for large tables HBM (the old entries in, the new ones out).  us in a graph: 10 rows of 9 pages 8, 320 rows of up to 64
// 12, 1021 rows of up to 2000 pages of a pool of 300 000 21
// (4 for the old counts, 4 for the new ones' zeros, by the eight CTAs that share them).
//
// One launch.  Every CTA works out for itself which children are heirs and which page a copy gets (a few bytes a row, from L2, and
// one sum over the rows) instead of waiting for another launch.  The first CTA, or for many pages a cluster of eight, then makes the counts
// and the free list, in phases with its barrier between them; the others write the rows, a warp some hundred entries.
// An old row and the child that counts for it cancel: only the entries that a row gains or loses touch a count.
#include <algorithm>

#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kPiece = 512;   // entries of a row that a warp writes
constexpr int kMaxPages = 1 << 26;

struct ForkArgs {
  int n_old, n_new, width, page, n_pages, most_free;   // most_free: what the free list has room for
  bool wide;   // counts at multiples of 16 bytes
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

// kCluster: CTAs that make the counts (and those of every cluster).
template <int kCluster>
__global__ void __launch_bounds__(kThreads, 1) fork_pages_kernel(const __grid_constant__ ForkArgs a) {
  extern __shared__ __align__(16) unsigned char raw[];
  unsigned long long* heir = reinterpret_cast<unsigned long long*>(raw);   // [n_old] (len, ~j) of its best child, 0: none
  int* copy = reinterpret_cast<int*>(heir + a.n_old);                     // [n_new] which of the copies it is
  __shared__ int s_sum[kWarps], s_count[8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = kCluster > 1 ? (int)cluster_ctarank() : 0;
  const auto sync_all = [] {   // of the CTAs that make the counts
    if constexpr (kCluster > 1) cluster_sync();
    else __syncthreads();
  };
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
  const int n_free = min(a.most_free, max(0, __ldg(a.n_free))), used = a.used ? min(n_free, max(0, __ldg(a.used))) : 0;

  if (blockIdx.x < kCluster) {   // the old counts, under way meanwhile
    const int step = kCluster * kThreads, first = rank * kThreads + tid, n4 = a.wide ? a.n_pages / 4 : 0;
#pragma unroll 8
    for (int p = first; p < n4; p += step) reinterpret_cast<int4*>(a.new_ref)[p] = __ldg(reinterpret_cast<const int4*>(a.ref) + p);
#pragma unroll 4
    for (int p = 4 * n4 + first; p < a.n_pages; p += step) a.new_ref[p] = __ldg(a.ref + p);
  }
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

  if (blockIdx.x >= kCluster) {   // rows, a warp a piece of one
    const int warps = (gridDim.x - kCluster) * kWarps, pieces = (a.width + kPiece - 1) / kPiece;
    for (long long it = (blockIdx.x - kCluster) * kWarps + warp; it < (long long)a.n_new * pieces; it += warps) {
      const int j = (int)(it / pieces), i0 = (int)(it % pieces) * kPiece + lane, i1 = min(a.width, i0 - lane + kPiece);
      const Child c = child_of(a, j);
      const int k = copy[j];
      const bool served = c.state == ATSPEED_PLAN_OK && k != kNoPage;
      const int kept = served ? c.kept : 0, fresh = k >= 0 ? fresh_page(j) : -1;
      const int* from = a.table + (long long)max(0, c.parent) * a.width;
      int* to = a.new_table + (long long)j * a.width;
      const int own = k >= 0 ? kept - 1 : kept;   // entries from the parent
#pragma unroll 8
      for (int i = i0; i < i1; i += 32) {
        int e = i < kept ? fresh : -1;
        if (i < own) e = __ldg(from + i);
        to[i] = e;
      }
      if (i0 == 0) {
        a.new_len[j] = served ? c.len : -1;
        a.new_state[j] = c.state != ATSPEED_PLAN_OK ? c.state : served ? ATSPEED_PLAN_OK : ATSPEED_PLAN_NO_PAGES;
        a.src[j] = k >= 0 ? last_entry(c) : -1;
        a.dst[j] = fresh;
      }
    }
    return;
  }
  // counts: what changes
  sync_all();   // (the old ones are there)
  const auto add = [&](int e, int v) {
    if (in_pool(e)) atomicAdd(a.new_ref + e, v);
  };
  for (int i = rank * kThreads + tid; i < used; i += kCluster * kThreads) add(__ldg(a.free + i), 1);
  // New rows, then old ones that no heir counts for: a lane finds out about one, the warp walks through their entries.
  // (entries i0 .. i1 of row p get v; what a warp does one after the other here is a chain of four reads a row)
  const int my_warp = rank * kWarps + warp, all_warps = kCluster * kWarps;
  const auto walk = [&](int p, int i0, int i1, int v) {
    unsigned rows = __ballot_sync(0xffffffffu, i0 < i1);
    while (rows) {
      int e[4], from[4], to[4], by[4], at[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int l = rows ? __ffs(rows) - 1 : 0;
        from[q] = __shfl_sync(0xffffffffu, i0, l) + lane, to[q] = rows ? __shfl_sync(0xffffffffu, i1, l) : 0;
        by[q] = __shfl_sync(0xffffffffu, v, l), at[q] = __shfl_sync(0xffffffffu, p, l);
        rows &= rows - 1;
        e[q] = from[q] < to[q] ? __ldg(a.table + (long long)at[q] * a.width + from[q]) : -1;
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) add(e[q], by[q]);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll 8
        for (int i = from[q] + 32; i < to[q]; i += 32) add(__ldg(a.table + (long long)at[q] * a.width + i), by[q]);
    }
  };
  for (int j0 = my_warp; j0 < a.n_new; j0 += 32 * all_warps) {
    const int j = j0 + lane * all_warps;
    int p = 0, from = 0, to = 0, v = 1;
    if (j < a.n_new) {
      const Child c = child_of(a, j);
      if (c.parent >= 0 && c.state == ATSPEED_PLAN_OK && copy[j] != kNoPage) {
        const int kept = c.kept - (copy[j] >= 0);
        p = c.parent, to = kept;
        if (is_heir(c, j)) from = kept, to = held_pages(a, p), v = -1;   // (with its parent's own hold)
        if (copy[j] >= 0) add(fresh_page(j), 1);
      }
    }
    walk(p, from, to, v);
  }
  for (int p0 = my_warp; p0 < a.n_old; p0 += 32 * all_warps) {
    const int p = p0 + lane * all_warps;
    const bool own = p < a.n_old && !(heir[p] && copy[~(uint32_t)heir[p]] != kNoPage);
    walk(p, 0, own ? held_pages(a, p) : 0, -1);
  }
  sync_all();
  // the free list: every warp a range of pages, in order, 128 at a time; which of them are free stays in a lane's bits
  constexpr int kHeld = 16;
  const int steps = (int)((a.n_pages + 128ll * kWarps * kCluster - 1) / (128ll * kWarps * kCluster));
  const long long p0 = 128ll * steps * (rank * kWarps + warp) + 4 * lane;   // the lane's first four
  const auto free_of = [&](int step) {
    const long long p = p0 + 128ll * step;
    uint32_t bits = 0;
    if (a.wide && p + 4 <= a.n_pages) {
      const int4 n = __ldcg(reinterpret_cast<const int4*>(a.new_ref + p));
      return (n.x <= 0 ? 1u : 0u) | (n.y <= 0 ? 2u : 0u) | (n.z <= 0 ? 4u : 0u) | (n.w <= 0 ? 8u : 0u);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) bits |= (p + i < a.n_pages && __ldcg(a.new_ref + p + i) <= 0 ? 1u : 0u) << i;
    return bits;
  };
  unsigned long long held = 0;
  int zeros = 0;
#pragma unroll 8
  for (int t = 0; t < steps; ++t) {
    const uint32_t bits = free_of(t);
    if (t < kHeld) held |= (unsigned long long)bits << 4 * t;
    zeros += __popc(bits);
  }
  zeros = __reduce_add_sync(0xffffffffu, zeros);
  int at = scan(lane == 0 ? zeros : 0, all), total = all;   // (lane 0's is the warp's)
  at = __shfl_sync(0xffffffffu, at, 0);
  if constexpr (kCluster > 1) {
    if (tid < kCluster)
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa_u32(&s_count[rank], tid)), "r"(all) : "memory");
    cluster_sync();
    total = 0;
    for (int r = 0; r < kCluster; ++r) {
      at += r < rank ? s_count[r] : 0;
      total += s_count[r];
    }
  }
  for (int t = 0; t < steps; ++t) {
    const uint32_t bits = t < kHeld ? (uint32_t)(held >> 4 * t) & 15u : free_of(t);
    if (!__any_sync(0xffffffffu, bits)) continue;
    // (the lanes' pages in order: those of the lanes before, then the lane's own)
    const unsigned before = (1u << lane) - 1u;
    int to = at;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned same = __ballot_sync(0xffffffffu, bits >> i & 1);
      to += __popc(same & before);
      at += __popc(same);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (bits >> i & 1) a.new_free[to++] = (int)(p0 + 128ll * t + i);
  }
  // -1 behind the free pages: up to a multiple of 16 bytes one by one, then by vectors
  int* rest = a.new_free + total;
  const int left = a.n_pages - total, me = rank * kThreads + tid;
  const int head = min(left, (int)((16 - (reinterpret_cast<uintptr_t>(rest) & 15)) & 15) / 4), vectors = (left - head) / 4;
  if (me < head) rest[me] = -1;
  for (int i = me; i < vectors; i += kCluster * kThreads) reinterpret_cast<int4*>(rest + head)[i] = make_int4(-1, -1, -1, -1);
  if (me < left - head - 4 * vectors) rest[head + 4 * vectors + me] = -1;
  if (rank == 0 && tid == 0) *a.new_n_free = total;
  if constexpr (kCluster > 1) cluster_sync();   // (no CTA leaves while others may write to its counts)
}

// Whether an output shares memory with an input or with another output (CTAs read inputs while others write).
bool overlapping(const atspeed_page_fork& f) {
  const long long o = 4ll * f.n_old, m = 4ll * f.n_new, pages = 4ll * f.n_pages;   // bytes; of a free list of unknown length its first entry's
  const Span in[] = {{f.d_table, o * f.table_width}, {f.d_kv_len, o}, {f.d_q_len, o}, {f.d_old_state, o}, {f.d_parent, m}, {f.d_length, m},
                     {f.d_ref, pages}, {f.d_free, f.free_size < 0 ? 0 : 4ll * std::max(1, f.free_size)}, {f.d_n_free, 4}, {f.d_used, 4}};
  const Span out[] = {{f.d_new_table, m * f.table_width}, {f.d_new_len, m}, {f.d_new_state, m}, {f.d_src, m}, {f.d_dst, m}, {f.d_new_ref, pages},
                      {f.d_new_free, pages}, {f.d_new_n_free, 4}};
  return outputs_overlap(out, in);
}

}  // namespace
}  // namespace atspeed

using namespace atspeed;

extern "C" atspeed_status atspeed_op_fork_pages(atspeed_stream stream, const atspeed_page_fork* fork) {
  if (!fork) return ATSPEED_E_ARG;
  const atspeed_page_fork& f = *fork;
  const int n_old = f.n_old, n_new = f.n_new, n_pages = f.n_pages, table_width = f.table_width;
  if (!f.d_table || !f.d_kv_len || !f.d_ref || !f.d_free || !f.d_n_free || !f.d_new_table || !f.d_new_len || !f.d_new_state || !f.d_src ||
      !f.d_dst || !f.d_new_ref || !f.d_new_free || !f.d_new_n_free || n_old <= 0 || n_new <= 0 || table_width <= 0 || f.page_size <= 0 ||
      n_pages <= 0)
    return ATSPEED_E_ARG;
  if (!f.d_parent && n_old != n_new) return ATSPEED_E_ARG;
  if (n_old > kMaxRequests || n_new > kMaxRequests || n_pages > kMaxPages || table_width > 0x7fffffff - kPiece) return ATSPEED_E_SHAPE;
  if (overlapping(f)) return ATSPEED_E_ARG;
  const int most_free = f.free_size ? std::max(0, f.free_size) : 0x7fffffff;
  const ForkArgs a = {n_old,     n_new,        table_width, f.page_size,   n_pages,       most_free,  aligned16(f.d_ref) && aligned16(f.d_new_ref),
                      f.d_table, f.d_kv_len,   f.d_q_len,   f.d_old_state, f.d_parent,    f.d_length, f.d_ref,
                      f.d_free,  f.d_n_free,   f.d_used,    f.d_new_table, f.d_new_len,   f.d_new_state, f.d_src,
                      f.d_dst,   f.d_new_ref,  f.d_new_free, f.d_new_n_free};
  const int smem = n_old * (int)sizeof(unsigned long long) + n_new * (int)sizeof(int);
  // Rows by as many CTAs as there is work for, up to the SMs that are left.  One CTA makes the counts of few pages and rows.
  const long long warps = (long long)n_new * ((table_width + kPiece - 1) / kPiece);
  const int writers = (int)std::min(136LL, (warps + kWarps - 1) / kWarps);
  static std::atomic<unsigned long long> done[2];
  if (n_pages <= 16384 && n_old + n_new <= 128) {
    if (smem_attr_once(done[0], fork_pages_kernel<1>, kMaxRequests * 12) != cudaSuccess) return ATSPEED_E_CUDA;
    fork_pages_kernel<1><<<1 + writers, kThreads, smem, (cudaStream_t)stream>>>(a);
    return launch_status();
  }
  if (smem_attr_once(done[1], fork_pages_kernel<8>, kMaxRequests * 12) != cudaSuccess) return ATSPEED_E_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(8 + (writers + 7) / 8 * 8), cfg.blockDim = dim3(kThreads), cfg.dynamicSmemBytes = smem, cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 8, attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr, cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, fork_pages_kernel<8>, a) == cudaSuccess ? ATSPEED_OK : ATSPEED_E_CUDA;
}
