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
constexpr float kLog2e = 1.4426950408889634f;

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
  double* lse;   // [R] log s, in 64 bits
  float* top;    // [R] m
};

// Order-preserving maps to whole numbers.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
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
  static __device__ __forceinline__ float at(const void* p, long long i) {
    float x;
    if constexpr (TYPE == ATSPEED_F32) x = __ldcs(static_cast<const float*>(p) + i);
    else x = unpack2(__ldcs(static_cast<const uint16_t*>(p) + i), TYPE == ATSPEED_F16).x;
    constexpr float most = TYPE == ATSPEED_F32 ? 3.40282347e38f : TYPE == ATSPEED_BF16 ? 3.38953139e38f : 65504.f;
    return x == x ? fminf(x, most) : -INFINITY;
  }
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

template <int TYPE>
__global__ void __launch_bounds__(kThreads) beam_pieces_kernel(const __grid_constant__ SelectArgs a) {
  constexpr int N = In<TYPE>::N;
  __shared__ Shared sh;
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cu0 = __ldg(a.cu), cu1 = __ldg(a.cu + a.n_req);
  if (row < cu0 || row >= cu1 || (a.final && __ldg(a.final + row) >= 0)) return;   // (the other kernel knows as much)
  const int st = a.state ? __ldg(a.state + row) : -1;
  const uint32_t* allowed = st >= 0 && st < a.n_states ? a.grammar + st * a.grammar_stride : nullptr;
  const bool nothing = st >= a.n_states && a.state;
  const int begin = piece * a.span, end = min(a.V, begin + a.span);
  const char* in = static_cast<const char*>(a.logits) + (long long)row * a.ld * (16 / N);
  if (tid == 0) sh.n = 0;
  float m = -INFINITY, s = 0.f;   // the thread's maximum and sum
  uint32_t floor = kNone;         // only what is above it is a candidate
  bool open = true;               // .. and fewer than W are known at or above a bound
  __syncthreads();
  for (int t0 = begin; t0 < end; t0 += kTile) {
    float x[kPer];   // token t0 + (i / N * kThreads + tid) * N + i % N
    const auto token = [&](int i) { return t0 + (i / N * kThreads + tid) * N + i % N; };
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = token(i) < end ? In<TYPE>::at(in, token(i)) : -INFINITY;
    uint32_t ok = 0xffffffffu;   // bit i: token(i) is allowed
    if (allowed) {
      ok = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (token(i) < end) ok |= (__ldg(allowed + (token(i) >> 5)) >> (token(i) & 31) & 1) << i;
    } else if (nothing) {
      ok = 0;
    }
    if (!a.full) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (!(ok >> i & 1)) x[i] = -INFINITY;
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) top = fmaxf(top, x[i]);
    if (top > m) {
      s *= exp2f((m - top) * kLog2e);
      m = top;
    }
    if (m > -INFINITY) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) s += exp2f((x[i] - m) * kLog2e);
    }
    if (a.full) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (!(ok >> i & 1)) x[i] = -INFINITY;
    }
    uint32_t k[kPer], from = floor + 1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) k[i] = key_of(x[i]);
    if (open) {   // from the W-th of the groups' maxima on
      if (a.W <= kThreads / 4) {
        uint32_t g = k[0];
#pragma unroll
        for (int i = 1; i < kPer; ++i) g = max(g, k[i]);
        sh.group[tid] = g;
        __syncthreads();
        uint32_t e[kThreads / 32];
#pragma unroll
        for (int i = 0; i < kThreads / 32; ++i) e[i] = sh.group[i * 32 + lane];
        from = max(from, warp_threshold(e, a.W, a.W + a.W / 4));
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t g = k[q];
#pragma unroll
          for (int i = 1; i < kPer / 4; ++i) g = max(g, k[4 * i + q]);
          sh.group[q * kThreads + tid] = g;
        }
        __syncthreads();
        uint32_t e[4 * kThreads / 32];
#pragma unroll
        for (int i = 0; i < 4 * kThreads / 32; ++i) e[i] = sh.group[i * 32 + lane];
        from = max(from, warp_threshold(e, a.W, a.W + a.W / 4));
      }
    }
    const int had = sh.n;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (k[i] >= from) {
        const int at = atomicAdd(&sh.n, 1);
        if (at < kList) {
          sh.key[at] = k[i];
          sh.tok[at] = token(i);
        }
      }
    __syncthreads();
    if (sh.n > kList) {   // too many: the tile's W best exactly, equal ones in the tokens' order
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
  const float sum = warp_sum(m > -INFINITY ? s * exp2f((m - M) * kLog2e) : 0.f);
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

struct RankShared {
  unsigned long long score[kRankList], rest[kRankList];
  uint32_t tok[kRankList];
  uint32_t group[kRankThreads];
  int n;
  uint32_t from;
};

__device__ __forceinline__ double score_of(unsigned long long k) {
  return __longlong_as_double((long long)(k >> 63 ? k ^ 1ull << 63 : ~k));
}
__device__ __forceinline__ uint32_t short_key(unsigned long long score) {   // its order is the scores', with equal ones
  return key_of((float)score_of(score));
}

// How many of the list come before entry i of it.
__device__ __forceinline__ int rank_of(const RankShared& sh, int n, const Entry& e) {
  int r = 0;
  for (int j = 0; j < n; ++j) {
    const unsigned long long s = sh.score[j];
    if (s > e.score) ++r;
    else if (s == e.score && (sh.rest[j] > e.rest || (sh.rest[j] == e.rest && sh.tok[j] < e.tok))) ++r;
  }
  return r;
}

__global__ void __launch_bounds__(kRankThreads) beam_rank_kernel(const __grid_constant__ SelectArgs a) {
  extern __shared__ __align__(16) unsigned char raw[];
  RankShared& sh = *reinterpret_cast<RankShared*>(raw);
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
  const int r0 = max(max(0, __ldg(a.cu)), __ldg(a.cu + b));
  const int r1 = min(min(a.R, __ldg(a.cu + a.n_req)), __ldg(a.cu + b + 1));
  const int lists = max(0, r1 - r0) * a.pieces;
  pdl_wait();
  for (int r = r0 + tid; r < r1; r += kRankThreads) {   // log s of the rows
    if (a.final && __ldg(a.final + r) >= 0) continue;
    float M = -INFINITY;
    for (int p = 0; p < a.pieces; ++p) M = fmaxf(M, a.head[(long long)r * a.pieces + p].m);
    double s = 0.0;
    for (int p = 0; p < a.pieces; ++p) {
      const Header h = a.head[(long long)r * a.pieces + p];
      if (h.m > -INFINITY) s += (double)h.s * exp((double)h.m - (double)M);
    }
    a.top[r] = M;
    a.lse[r] = log(s);
  }
  if (tid == 0) sh.n = 0;
  __syncthreads();
  const long long slots = (long long)lists * a.cap;
  // candidate i of the request, if there is one (an ended beam has one, in the first place of its first piece)
  const auto get = [&](long long i, Entry& e) {
    const int l = (int)(i / a.cap), at = (int)(i % a.cap), r = r0 + l / a.pieces;
    const double cum = a.score ? (double)__ldg(a.score + r) : 0.0;
    double score;
    float x = 0.f;
    const int end = a.final ? __ldg(a.final + r) : -1;
    if (end >= 0) {
      if (at || l % a.pieces) return false;
      score = cum;
      e.tok = (uint32_t)end;
    } else {
      const long long h = (long long)r0 * a.pieces + l;
      if (at >= a.head[h].n) return false;
      const uint2 c = a.cand[h * a.cap + at];
      x = __uint_as_float(c.x);
      e.tok = c.y;
      score = cum + (((double)x - (double)a.top[r]) - a.lse[r]);
    }
    if (!((float)score > -INFINITY)) return false;
    e.score = key_of(score + 0.0);   // (-0: 0)
    e.rest = (unsigned long long)(~(uint32_t)r) << 32 | key_of(x);
    return true;
  };
  uint32_t from = kNone + 1;
  Entry e;
  if (slots > kRankList) {   // more than the list holds: from the W-th of the threads' best on
    uint32_t g = 0;
    for (long long i = tid; i < slots; i += kRankThreads)
      if (get(i, e)) g = max(g, short_key(e.score));
    sh.group[tid] = g;
    __syncthreads();
    if (tid < 32) {
      uint32_t k[kRankThreads / 32];
#pragma unroll
      for (int i = 0; i < kRankThreads / 32; ++i) k[i] = sh.group[i * 32 + lane];
      const uint32_t t = warp_threshold(k, a.W, a.W + a.W / 4);
      if (lane == 0) sh.from = t;
    }
    __syncthreads();
    from = sh.from;
  }
  for (long long i0 = 0; i0 < slots; i0 += kRankThreads) {
    if (i0 + tid < slots && get(i0 + tid, e) && short_key(e.score) >= from) {
      const int at = atomicAdd(&sh.n, 1);
      sh.score[at] = e.score;
      sh.rest[at] = e.rest;
      sh.tok[at] = e.tok;
    }
    __syncthreads();
    const int n = sh.n;
    if (n > kRankList - kRankThreads && i0 + kRankThreads < slots) {   // the W best stay
      Entry mine[kRankList / kRankThreads];
      int r[kRankList / kRankThreads];
#pragma unroll
      for (int q = 0; q < kRankList / kRankThreads; ++q) {
        const int j = q * kRankThreads + tid;
        r[q] = a.W;
        if (j < n) {
          mine[q] = {sh.score[j], sh.rest[j], sh.tok[j]};
          r[q] = rank_of(sh, n, mine[q]);
        }
      }
      __syncthreads();
#pragma unroll
      for (int q = 0; q < kRankList / kRankThreads; ++q)
        if (r[q] < a.W) {
          sh.score[r[q]] = mine[q].score;
          sh.rest[r[q]] = mine[q].rest;
          sh.tok[r[q]] = mine[q].tok;
        }
      if (tid == 0) sh.n = min(n, a.W);
      __syncthreads();
      if (n >= a.W) from = max(from, short_key(sh.score[a.W - 1]));
    }
    __syncthreads();
  }
  const int n = sh.n;
  const long long o = (long long)b * a.W;
  for (int j = tid; j < n; j += kRankThreads) {
    const Entry x = {sh.score[j], sh.rest[j], sh.tok[j]};
    const int r = rank_of(sh, n, x);
    if (r < a.W) {
      a.token[o + r] = (int)x.tok;
      a.parent[o + r] = (int)~(uint32_t)(x.rest >> 32);
      a.out_score[o + r] = (float)score_of(x.score);
    }
  }
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
int cap_of(int W) { return W + W / 2 + 16; }

struct Layout {
  int pieces;
  size_t cand, lse, top, bytes;
};
Layout layout_of(int R, int V, int W) {
  Layout l;
  l.pieces = pieces_of(R, V);
  const size_t n = (size_t)R * l.pieces;
  l.cand = n * sizeof(Header);
  l.lse = l.cand + n * cap_of(W) * sizeof(uint2);
  l.top = l.lse + (size_t)R * sizeof(double);
  l.bytes = l.top + (size_t)R * sizeof(float);
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
  a.lse = reinterpret_cast<double*>(ws + l.lse), a.top = reinterpret_cast<float*>(ws + l.top);
  static std::atomic<unsigned long long> done{0};
  if (smem_attr_once(done, beam_rank_kernel, (int)sizeof(RankShared)) != cudaSuccess) return ATSPEED_E_CUDA;
  const int grid = R * l.pieces;
  if (type == ATSPEED_F32) beam_pieces_kernel<ATSPEED_F32><<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
  else if (type == ATSPEED_BF16) beam_pieces_kernel<ATSPEED_BF16><<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
  else beam_pieces_kernel<ATSPEED_F16><<<grid, kThreads, 0, (cudaStream_t)stream>>>(a);
  beam_rank_kernel<<<n_req, kRankThreads, sizeof(RankShared), (cudaStream_t)stream>>>(a);
  return launch_status();
}
