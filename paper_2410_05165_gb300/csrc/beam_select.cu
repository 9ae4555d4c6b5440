// Beam search's selection over beams and vocabulary (atspeed_op_beam_select).
//   score(r, v) = cum_r + ((x_rv - m_r) - log s_r),  m_r = max x_r,  s_r = sum_v exp(x_rv - m_r);  the best W of a request's rows
// Bound: HBM (each logit read once).
//
// Two launches.  The first reads the logits, a CTA a piece of a row: the piece's maximum, its sum of exponentials and the
// candidates among its logits, which are at least its W best (within a row the order is the logits').  The second, a CTA a
// request, makes log s_r of the pieces, scores the candidates in 64 bits and ranks the best.
//
// Candidates of a piece: W of the largest values of 256 (1024) groups of its first tile lie at or above the W-th largest group maximum, so what is
// below it is none; behind that tile only what is above it.  What is left goes to a list in shared memory, that is cut to
// the W best when it is half full.  A tile that holds more than fits (equal logits, a mask of the type's lowest value) is
// searched exactly.
//
// Sums of a row do not depend on where the row begins in memory: rows with the same logits have the same bits.
#include <algorithm>

#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kPer = 16;                    // logits of a thread in a tile
constexpr int kTile = kThreads * kPer;
constexpr int kList = 1024;                 // candidates that a piece's list holds
constexpr int kMaxWidth = 256;
constexpr int kRankThreads = 1024, kRankList = 2048;
constexpr uint32_t kNone = 0x007fffffu;     // the key of -infinity

struct Header {   // of a piece
  float m, s;
  int n;
  int pad;
};

struct SelectArgs {
  const void* logits;
  long long ld;
  int R, V, n_req, W, pieces, span, cap;   // span: tokens of a piece, cap: candidates it hands on
  const float* score;
  const int *final, *cu, *state;
  const uint32_t* grammar;
  long long grammar_stride;
  int n_states;
  bool full;
  int *token, *parent;
  float* out_score;
  Header* head;
  uint2* cand;   // (logit, token)
  struct Row* rows;   // [R]
};

// Order-preserving maps to whole numbers.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);   // (-0: 0)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ unsigned long long key_of(double x) {
  const unsigned long long b = (unsigned long long)__double_as_longlong(x);
  return b >> 63 ? ~b : b | 1ull << 63;
}

template <int TYPE>
struct In {
  static constexpr int N = TYPE == ATSPEED_F32 ? 4 : 8;   // logits of 16 bytes
};

// The largest t with at least `want` of the warp's keys (E a lane, all valid ones above kNone) at or above it, or a
// smaller one with at most `most` there; kNone + 1 where there are fewer than `want`.
template <int E>
__device__ uint32_t warp_threshold(const uint32_t (&k)[E], int want, int most) {
  uint32_t lo = 0xffffffffu, hi = 0;
  int valid = 0;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (k[e] > kNone) lo = min(lo, k[e]), hi = max(hi, k[e]), ++valid;
  valid = __reduce_add_sync(0xffffffffu, valid);
  if (valid < want) return kNone + 1;
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (valid <= most) return lo;
  while (lo < hi) {   // at least `want` at lo, fewer above hi
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    int c = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) c += k[e] >= mid;
    c = __reduce_add_sync(0xffffffffu, c);
    if (c >= want) {
      lo = mid;
      if (c <= most) break;
    } else {
      hi = mid - 1;
    }
  }
  return lo;
}

struct Shared {
  uint32_t key[kList];
  int tok[kList];
  uint32_t group[4 * kThreads];
  int n, count[kWarps];
  float m[kWarps], s[kWarps];
};

__device__ __forceinline__ int block_count(int v, Shared& sh) {   // the sum over the CTA
  v = __reduce_add_sync(0xffffffffu, v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh.count[threadIdx.x >> 5] = v;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) t += sh.count[w];
  return t;
}

// Cuts the list to its W best (equal keys: the lower tokens); returns the W-th key.  Every thread of the CTA.
__device__ uint32_t cut_list(Shared& sh, int W) {
  constexpr int E = kList / kThreads;
  const int n = sh.n;
  uint32_t k[E];
  int t[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = e * kThreads + threadIdx.x;
    k[e] = i < n ? sh.key[i] : 0u;
    t[e] = i < n ? sh.tok[i] : 0;
  }
  uint32_t lo = kNone + 1, hi = 0xffffffffu;
  while (lo < hi) {   // (n > W: at least W at lo)
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    int c = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) c += k[e] >= mid;
    if (block_count(c, sh) >= W) lo = mid;
    else hi = mid - 1;
  }
  int above = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) above += k[e] > lo;
  above = block_count(above, sh);
  // of the keys at lo, those with fewer than W - above lower tokens
  bool keep[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    keep[e] = k[e] > lo;
    if (k[e] == lo) {
      int before = 0;
      for (int i = 0; i < n; ++i) before += sh.key[i] == lo && sh.tok[i] < t[e];
      keep[e] = above + before < W;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) sh.n = 0;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (keep[e]) {
      const int at = atomicAdd(&sh.n, 1);
      sh.key[at] = k[e];
      sh.tok[at] = t[e];
    }
  __syncthreads();
  return lo;
}

// A sum of exponentials below a maximum m: for |m| < kFar in units of the whole power of two 2^unit_of(m), its terms 2^(x l - unit)
// by one multiply-add (l = log2 e in 32 bits), so that another maximum rescales it exactly, whatever their order; from
// kFar on, where x l has no bits left for that, in units of e^m.
// e^x as 2^(x l) is off by a factor e^(x kEta), which the scores take back for the row's maximum.
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.69314718055994530942, kEta = (double)kLog2e * kLn2 - 1.0;
constexpr float kFar = 0x1p20f;

__device__ __forceinline__ float unit_of(float m) { return rintf(m * kLog2e); }
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// What a sum below m is worth below M >= m.
__device__ __forceinline__ float rescale(float m, float M) {
  if (m == M) return 1.f;
  const bool near = fabsf(m) < kFar, NEAR = fabsf(M) < kFar;
  return exp2_approx(near ? NEAR ? unit_of(m) - unit_of(M) : fmaf(-M, kLog2e, unit_of(m))
                          : NEAR ? fmaf(m, kLog2e, -unit_of(M)) : (m - M) * kLog2e);
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads) beam_pieces_kernel(const __grid_constant__ SelectArgs a) {
  constexpr int N = In<TYPE>::N, SIZE = 16 / N;
  __shared__ Shared sh;
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch_dependents();
  const int cu0 = __ldg(a.cu), cu1 = __ldg(a.cu + a.n_req);
  if (row < cu0 || row >= cu1 || (a.final && __ldg(a.final + row) >= 0)) return;   // (the other kernel knows as much)
  const int st = a.state ? __ldg(a.state + row) : -1;
  const uint32_t* allowed = st >= 0 && st < a.n_states ? a.grammar + st * a.grammar_stride : nullptr;
  const bool nothing = st >= a.n_states && a.state;
  const int begin = piece * a.span, end = min(a.V, begin + a.span);
  const char* in = static_cast<const char*>(a.logits) + (long long)row * a.ld * SIZE;
  const unsigned lead = (unsigned)(reinterpret_cast<uintptr_t>(in) & 15);   // bytes that the row begins behind a 16-byte word
  if (tid == 0) sh.n = 0;
  float m = -INFINITY, s = 0.f;   // the thread's maximum and sum
  uint32_t floor = kNone;         // only what is above it is a candidate
  bool open = true;               // .. and fewer than W are known at or above a bound
  __syncthreads();
  for (int t0 = begin; t0 < end; t0 += kTile) {
    float x[kPer];   // token t0 + (i / N * kThreads + tid) * N + i % N
    const auto token = [&](int i) { return t0 + (i / N * kThreads + tid) * N + i % N; };
    // A thread's logits of a vector, wherever the row begins: the 16-byte words that they lie in, shifted.  At the row's ends one by one.
    uint4 w[kPer / N];
    if (t0 + kTile <= end && lead == 0) {
#pragma unroll
      for (int v = 0; v < kPer / N; ++v) w[v] = __ldcs(reinterpret_cast<const uint4*>(in + (long long)token(v * N) * SIZE));
    } else {
#pragma unroll
      for (int v = 0; v < kPer / N; ++v) {
        const int t = token(v * N);
        const char* at = in + (long long)t * SIZE - lead;
        if (t + 2 * N <= a.V && t + N <= end && t > 0) {
          const uint4 p = __ldg(reinterpret_cast<const uint4*>(at));
          w[v] = p;
          if (lead) {
            const uint4 q = __ldg(reinterpret_cast<const uint4*>(at) + 1);
            uint32_t y[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
            if (lead & 8) {
#pragma unroll
              for (int j = 0; j < 6; ++j) y[j] = y[j + 2];
            }
            if (lead & 4) {
#pragma unroll
              for (int j = 0; j < 5; ++j) y[j] = y[j + 1];
            }
            if (SIZE == 2 && (lead & 2)) {
#pragma unroll
              for (int j = 0; j < 4; ++j) y[j] = __funnelshift_r(y[j], y[j + 1], 16);
            }
            w[v] = make_uint4(y[0], y[1], y[2], y[3]);
          }
        } else {
          uint32_t y[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (SIZE == 4) {
              y[j] = t + j < end ? __ldg(reinterpret_cast<const uint32_t*>(in) + t + j) : 0xff800000u;
            } else {
              const uint16_t* h = reinterpret_cast<const uint16_t*>(in);
              const uint32_t none = TYPE == ATSPEED_F16 ? 0xfc00u : 0xff80u;
              const uint32_t lo = t + 2 * j < end ? __ldg(h + t + 2 * j) : none, hi = t + 2 * j + 1 < end ? __ldg(h + t + 2 * j + 1) : none;
              y[j] = lo | hi << 16;
            }
          }
          w[v] = make_uint4(y[0], y[1], y[2], y[3]);
        }
      }
    }
#pragma unroll
    for (int v = 0; v < kPer / N; ++v) {
      const uint32_t y[4] = {w[v].x, w[v].y, w[v].z, w[v].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (SIZE == 4) {
          x[v * N + j] = __uint_as_float(y[j]);
        } else {
          const float2 f = unpack2(y[j], TYPE == ATSPEED_F16);
          x[v * N + 2 * j] = f.x;
          x[v * N + 2 * j + 1] = f.y;
        }
      }
    }
    uint32_t ok = 0xffffffffu;   // bit i: token(i) is allowed
    if (allowed) {
      ok = 0;
#pragma unroll
      for (int v = 0; v < kPer / N; ++v) {   // (a vector's bits lie in one word)
        const int t = token(v * N);
        if (t < end) ok |= (__ldg(allowed + (t >> 5)) >> (t & 31) & ((1u << N) - 1)) << v * N;
      }
    } else if (nothing) {
      ok = 0;
    }
    if (ok != 0xffffffffu && !a.full) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (!(ok >> i & 1)) x[i] = -INFINITY;
    }
    float top = x[0];   // (a NaN is passed over)
#pragma unroll
    for (int i = 1; i < kPer; ++i) top = fmaxf(top, x[i]);
    top = fmaxf(top, -INFINITY);
    float sum = 0.f, M = fmaxf(m, top);
    if (M > -INFINITY) {
      if (fabsf(M) < kFar) {
        const float u = unit_of(M);
#pragma unroll
        for (int i = 0; i < kPer; ++i) sum += exp2_approx(fmaf(x[i], kLog2e, -u));
      } else {
        sum = NAN;
      }
      if (sum != sum) {   // a NaN (it counts as -infinity), an infinity (as the type's largest), logits far out
        constexpr float most = TYPE == ATSPEED_F32 ? 3.40282347e38f : TYPE == ATSPEED_BF16 ? 3.38953139e38f : 65504.f;
        top = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          x[i] = x[i] == x[i] ? fminf(x[i], most) : -INFINITY;
          top = fmaxf(top, x[i]);
        }
        M = fmaxf(m, top);
        const bool near = fabsf(M) < kFar;
        const float u = unit_of(M);
        if (M > -INFINITY) {
#pragma unroll
          for (int i = 0; i < kPer; ++i) sum += exp2_approx(near ? fmaf(x[i], kLog2e, -u) : (x[i] - M) * kLog2e);
        }
      }
      if (M > m) {
        s = m > -INFINITY ? s * rescale(m, M) : 0.f;
        m = M;
      }
    }
    s += sum;
    if (ok != 0xffffffffu && a.full) {
      top = -INFINITY;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (!(ok >> i & 1)) x[i] = -INFINITY;
        top = fmaxf(top, x[i]);
      }
    }
    uint32_t from = floor + 1;
    if (open) {   // from the W-th of the groups' maxima on
      if (a.W <= kThreads / 4) {
        sh.group[tid] = key_of(top);
        __syncthreads();
        uint32_t e[kThreads / 32];
#pragma unroll
        for (int i = 0; i < kThreads / 32; ++i) e[i] = sh.group[i * 32 + lane];
        from = max(from, warp_threshold(e, a.W, a.W + a.W / 4));
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float g = x[q];
#pragma unroll
          for (int i = 1; i < kPer / 4; ++i) g = fmaxf(g, x[4 * i + q]);
          sh.group[q * kThreads + tid] = key_of(g);
        }
        __syncthreads();
        uint32_t e[4 * kThreads / 32];
#pragma unroll
        for (int i = 0; i < 4 * kThreads / 32; ++i) e[i] = sh.group[i * 32 + lane];
        from = max(from, warp_threshold(e, a.W, a.W + a.W / 4));
      }
    }
    const float least = value_of(from);
    const int had = sh.n;
    __syncthreads();
    if (top >= least) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (x[i] >= least) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < kList) {
            sh.key[at] = key_of(x[i]);
            sh.tok[at] = token(i);
          }
        }
    }
    __syncthreads();
    if (sh.n > kList) {   // too many: the tile's W best exactly, equal ones in the tokens' order
      uint32_t k[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) k[i] = x[i] >= least ? key_of(x[i]) : 0u;
      uint32_t lo = from, hi = 0xffffffffu;
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + 1;
        int c = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) c += k[i] >= mid;
        if (block_count(c, sh) >= a.W) lo = mid;
        else hi = mid - 1;
      }
      int above = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) above += k[i] > lo;
      int room = a.W - block_count(above, sh);   // for equal ones (at least one)
      __syncthreads();
      if (tid == 0) sh.n = had;
      __syncthreads();
      const auto put = [&](int i, int at) {
        sh.key[at] = k[i];
        sh.tok[at] = token(i);
      };
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (k[i] > lo) put(i, atomicAdd(&sh.n, 1));
      __syncthreads();
      int at0 = sh.n;
      // (a thread's tokens follow each other in its vectors, the vectors of all threads in the tile)
#pragma unroll
      for (int v = 0; v < kPer / N; ++v) {
        int mine = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) mine += k[v * N + j] == lo;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += y;
        }
        __syncthreads();
        if (lane == 31) sh.count[warp] = upto;
        __syncthreads();
        int nth = upto - mine, all = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          if (w < warp) nth += sh.count[w];
          all += sh.count[w];
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (k[v * N + j] == lo) {
            if (nth < room) put(v * N + j, at0 + nth);
            ++nth;
          }
        at0 += min(room, all);
        room -= min(room, all);
      }
      __syncthreads();
      if (tid == 0) sh.n = at0;
      __syncthreads();
    }
    if (open && from > kNone + 1) {   // (W of the tile's are at `from` or above: a later token there comes after them)
      open = false;
      floor = from;
    }
    if (sh.n > kList / 2) {
      open = false;
      floor = cut_list(sh, a.W);
    }
    __syncthreads();
  }
  if (sh.n > a.cap) cut_list(sh, a.W);
  const long long at = (long long)row * a.pieces + piece;
  for (int i = tid; i < sh.n; i += kThreads)
    a.cand[at * a.cap + i] = make_uint2(__float_as_uint(value_of(sh.key[i])), (uint32_t)sh.tok[i]);
  // the piece's sum, in one order
  float M = warp_max(m);
  if (lane == 0) sh.m[warp] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sh.m[w]);
  const float sum = warp_sum(m > -INFINITY ? s * rescale(m, M) : 0.f);
  if (lane == 0) sh.s[warp] = sum;
  __syncthreads();
  if (tid == 0) {
    float all = 0.f;
    for (int w = 0; w < kWarps; ++w) all += sh.s[w];
    a.head[at] = {M, all, sh.n, 0};
  }
}

// A candidate of a request: equal scores, the lower row first, then the larger logit, then the lower token.
struct Entry {
  unsigned long long score;   // (as an ordered key)
  unsigned long long rest;    // ~row, logit's key
  uint32_t tok;
};

// score = cum + ((x - off) - more)
struct Row {
  double off, more;
  float cum;
  int final;   // the one token of an ended beam; -1
};

constexpr int kRows = 256;   // that shared memory holds (of more: device memory)
struct RankShared {
  unsigned long long score[kRankList], rest[kRankList];
  uint32_t tok[kRankList];
  uint32_t group[kRankThreads];
  Row row[kRows];
  Entry best[kMaxWidth];
  int n;
  uint32_t from;
};

__device__ __forceinline__ double score_of(unsigned long long k) {
  return __longlong_as_double((long long)(k >> 63 ? k ^ 1ull << 63 : ~k));
}

// Ranks the list's n entries and hands each that is among the W best to put(rank, entry).  Every thread of the CTA; several threads
// an entry, neighbours in a warp.
template <class Put>
__device__ __forceinline__ void rank_list(const RankShared& sh, int n, int W, Put&& put) {
  int share = 32;   // threads an entry
  while (share > 1 && share * n > kRankThreads) share >>= 1;
  const int per = kRankThreads / share, sub = threadIdx.x % share;
  for (int j0 = 0; j0 < n; j0 += per) {
    const int j = j0 + threadIdx.x / share;
    Entry e = {0, 0, 0};
    if (j < n) e = {sh.score[j], sh.rest[j], sh.tok[j]};
    int r = 0;
    for (int i = sub; i < n; i += share) {
      const unsigned long long s = sh.score[i];
      if (s > e.score) ++r;
      else if (s == e.score && (sh.rest[i] > e.rest || (sh.rest[i] == e.rest && sh.tok[i] < e.tok))) ++r;
    }
    for (int o = share >> 1; o > 0; o >>= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
    if (j < n && sub == 0 && r < W) put(r, e);
  }
}

__global__ void __launch_bounds__(kRankThreads) beam_rank_kernel(const __grid_constant__ SelectArgs a) {
  extern __shared__ __align__(16) unsigned char raw[];
  RankShared& sh = *reinterpret_cast<RankShared*>(raw);
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r0 = max(max(0, __ldg(a.cu)), __ldg(a.cu + b));
  const int r1 = min(min(a.R, __ldg(a.cu + a.n_req)), __ldg(a.cu + b + 1));
  const int lists = max(0, r1 - r0) * a.pieces;
  if (tid == 0) sh.n = 0;
  pdl_wait();
  for (int r = r0 + tid; r < r1; r += kRankThreads) {
    Row w = {0.0, 0.0, a.score ? __ldg(a.score + r) : 0.f, a.final ? __ldg(a.final + r) : -1};
    if (w.final < 0) {
      const Header* h = a.head + (long long)r * a.pieces;
      float M = -INFINITY;
      for (int p = 0; p < a.pieces; ++p) M = fmaxf(M, h[p].m);
      double s = 0.0;
      for (int p = 0; p < a.pieces; ++p)
        if (h[p].m > -INFINITY) s += (double)(h[p].s * rescale(h[p].m, M));   
      const double l = log(s);
      if (fabsf(M) < kFar) w.off = (double)unit_of(M) * kLn2 + l - (double)M * kEta;
      else w.off = (double)M, w.more = l;
    }
    if (r - r0 < kRows) sh.row[r - r0] = w;
    else a.rows[r] = w;
  }
  __syncthreads();
  // Candidate `at` of list l, in 32 bits: between low and high.
  const int lists_at_once = kRankThreads / a.cap, at = tid % a.cap, my_list = tid / a.cap;
  struct Found {
    float x, low, high;
    uint32_t tok;
    int row;
  };
  const auto row_of = [&](int r) -> const Row& { return r - r0 < kRows ? sh.row[r - r0] : a.rows[r]; };
  const auto look = [&](int l, const uint2& c, int n, Found& f) {   // c, n: of that list
    f.row = r0 + l / a.pieces;
    const Row& w = row_of(f.row);
    if (w.final >= 0) {
      f.tok = (uint32_t)w.final, f.x = 0.f, f.low = f.high = w.cum;
      return at == 0 && l % a.pieces == 0;
    }
    f.x = __uint_as_float(c.x), f.tok = c.y;
    const float off = (float)w.off, more = (float)w.more;
    const float y = w.cum + ((f.x - off) - more), e = 0x1p-21f * (fabsf(w.cum) + fabsf(f.x) + fabsf(off) + fabsf(more));
    f.low = y - e, f.high = y + e;
    return at < n;
  };
  const auto fetch = [&](int l, uint2& c, int& n) {
    const long long h = (long long)r0 * a.pieces + l;
    c = a.cand[h * a.cap + at];
    n = a.head[h].n;
  };
  float from = -INFINITY;   // what is below it (in 32 bits) is not among the W best
  if (lists > lists_at_once) {   // more than a step's: from the W-th of the threads' best on
    float g = -INFINITY;
    for (int l = my_list; l < lists; l += 4 * lists_at_once) {
      uint2 c[4];
      int n[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (l + q * lists_at_once < lists) fetch(l + q * lists_at_once, c[q], n[q]);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        Found f;
        if (l + q * lists_at_once < lists && look(l + q * lists_at_once, c[q], n[q], f)) g = fmaxf(g, f.low);   // (not a NaN)
      }
    }
    sh.group[tid] = key_of(g);
    __syncthreads();
    if (warp == 0) {
      uint32_t k[kRankThreads / 32];
#pragma unroll
      for (int i = 0; i < kRankThreads / 32; ++i) k[i] = sh.group[i * 32 + lane];
      const uint32_t t = warp_threshold(k, a.W, a.W + a.W / 4);
      if (lane == 0) sh.from = t;
    }
    __syncthreads();
    if (sh.from > kNone + 1) from = value_of(sh.from);
  }
  for (int l0 = 0; l0 < lists; l0 += lists_at_once) {
    const int l = l0 + my_list;
    if (my_list < lists_at_once && l < lists) {
      uint2 c;
      int n;
      Found f;
      fetch(l, c, n);
      if (look(l, c, n, f) && !(f.high < from)) {
        const Row& w = row_of(f.row);
        const double y = w.final >= 0 ? (double)w.cum : (double)w.cum + (((double)f.x - w.off) - w.more);
        if ((float)y > -INFINITY) {
          const int to = atomicAdd(&sh.n, 1);
          sh.score[to] = key_of(y + 0.0);   // (-0: 0)
          sh.rest[to] = (unsigned long long)(~(uint32_t)f.row) << 32 | key_of(f.x);
          sh.tok[to] = f.tok;
        }
      }
    }
    if (l0 + lists_at_once >= lists) break;
    __syncthreads();
    const int n = sh.n;
    if (n > kRankList - kRankThreads) {   // the W best stay
      rank_list(sh, n, a.W, [&](int r, const Entry& e) { sh.best[r] = e; });
      __syncthreads();
      for (int j = tid; j < min(n, a.W); j += kRankThreads) sh.score[j] = sh.best[j].score, sh.rest[j] = sh.best[j].rest, sh.tok[j] = sh.best[j].tok;
      if (tid == 0) {
        sh.n = min(n, a.W);
        // (in 32 bits, rounded down)
        sh.from = n >= a.W ? key_of(__double2float_rd(score_of(sh.best[a.W - 1].score))) : 0u;
      }
      __syncthreads();
      if (sh.from) from = fmaxf(from, value_of(sh.from));
    }
    __syncthreads();
  }
  __syncthreads();
  const int n = sh.n;
  const long long o = (long long)b * a.W;
  rank_list(sh, n, a.W, [&](int r, const Entry& e) {
    a.token[o + r] = (int)e.tok;
    a.parent[o + r] = (int)~(uint32_t)(e.rest >> 32);
    a.out_score[o + r] = (float)score_of(e.score);
  });
  for (int j = n + tid; j < a.W; j += kRankThreads) {
    a.token[o + j] = -1;
    a.parent[o + j] = -1;
    a.out_score[o + j] = -INFINITY;
  }
}

// Pieces of a row: enough CTAs for every SM to have four, none shorter than a tile.
int pieces_of(int R, int V) {
  const long long tiles = (V + kTile - 1LL) / kTile;
  return (int)std::max(1LL, std::min(tiles, (608LL + R - 1) / R));
}
int cap_of(int W) {   
  int cap = 32;
  while (cap < W + std::max(8, W / 4)) cap *= 2;
  return cap;
}

struct Layout {
  int pieces;
  size_t cand, rows, bytes;
};
Layout layout_of(int R, int V, int W) {
  Layout l;
  l.pieces = pieces_of(R, V);
  const size_t n = (size_t)R * l.pieces;
  l.cand = n * sizeof(Header);
  l.rows = l.cand + n * cap_of(W) * sizeof(uint2);
  l.bytes = l.rows + (size_t)R * sizeof(Row);
  return l;
}

}  // namespace
}  // namespace atspeed

using namespace atspeed;

extern "C" size_t atspeed_op_beam_select_workspace(int R, int vocab, int width) {
  return R > 0 && vocab > 0 && width > 0 ? layout_of(R, vocab, std::min(width, kMaxWidth)).bytes : 0;
}

extern "C" atspeed_status atspeed_op_beam_select(atspeed_stream stream, const void* d_logits, atspeed_dtype type, int64_t ld, int R,
                                                 int vocab, const float* d_score, const int32_t* d_final, int n_req,
                                                 const int32_t* d_cu_beam, int width, const int32_t* d_state,
                                                 const uint32_t* d_grammar, int64_t grammar_stride, int n_states,
                                                 atspeed_norm_mode norm, int32_t* d_token, int32_t* d_parent,
                                                 float* d_out_score, void* d_ws) {
  if (!d_logits || !d_cu_beam || !d_token || !d_parent || !d_out_score || !d_ws || R <= 0 || vocab <= 0 || n_req <= 0 || width <= 0 ||
      ld < vocab || !dtype_size(type) || reinterpret_cast<uintptr_t>(d_logits) % dtype_size(type) || !aligned16(d_ws) ||
      (norm != ATSPEED_NORM_MASKED && norm != ATSPEED_NORM_FULL) ||
      (d_state && (!d_grammar || n_states <= 0 || grammar_stride < (vocab + 31LL) / 32)))
    return ATSPEED_E_ARG;
  const Layout l = layout_of(R, vocab, std::min(width, kMaxWidth));
  if (width > kMaxWidth || vocab > 1 << 30 || (long long)R * l.pieces > 0x7fffffffLL) return ATSPEED_E_SHAPE;
  SelectArgs a = {};
  a.logits = d_logits, a.ld = ld, a.R = R, a.V = vocab, a.n_req = n_req, a.W = width, a.pieces = l.pieces, a.cap = cap_of(width);
  a.span = (int)(((vocab + (long long)l.pieces - 1) / l.pieces + kTile - 1) / kTile * kTile);
  a.score = d_score, a.final = d_final, a.cu = d_cu_beam, a.state = d_state, a.grammar = d_grammar;
  a.grammar_stride = grammar_stride, a.n_states = d_state ? n_states : 0, a.full = norm == ATSPEED_NORM_FULL;
  a.token = d_token, a.parent = d_parent, a.out_score = d_out_score;
  char* ws = static_cast<char*>(d_ws);
  a.head = reinterpret_cast<Header*>(ws), a.cand = reinterpret_cast<uint2*>(ws + l.cand);
  a.rows = reinterpret_cast<Row*>(ws + l.rows);
  static std::atomic<unsigned long long> done{0};
  if (smem_attr_once(done, beam_rank_kernel, (int)sizeof(RankShared)) != cudaSuccess) return ATSPEED_E_CUDA;
  const int grid = R * l.pieces;
  if (type == ATSPEED_F32) beam_pieces_kernel<ATSPEED_F32><<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
  else if (type == ATSPEED_BF16) beam_pieces_kernel<ATSPEED_BF16><<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
  else beam_pieces_kernel<ATSPEED_F16><<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
  if (launch_status() != ATSPEED_OK) return ATSPEED_E_CUDA;
  // (it may start while the last of the pieces are read, and waits for them)
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_req), cfg.blockDim = dim3(kRankThreads), cfg.dynamicSmemBytes = sizeof(RankShared), cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr, cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, beam_rank_kernel, a) == cudaSuccess ? ATSPEED_OK : ATSPEED_E_CUDA;
}
