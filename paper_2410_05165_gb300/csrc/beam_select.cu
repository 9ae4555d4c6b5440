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
#include <type_traits>

#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kVec = 4;                     // 16-byte vectors of a thread in a tile
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
  static constexpr int SIZE = TYPE == ATSPEED_F32 ? 4 : 2, N = 16 / SIZE;   // N: logits of 16 bytes
  static constexpr int TILE = kThreads * kVec * N;
  static constexpr uint32_t NONE = TYPE == ATSPEED_F32 ? 0xff800000u : TYPE == ATSPEED_F16 ? 0xfc00u : 0xff80u;   // -infinity
  static constexpr uint32_t MOST = TYPE == ATSPEED_F32 ? 0x7f7fffffu : TYPE == ATSPEED_F16 ? 0x7bffu : 0x7f7fu;
  static __device__ __forceinline__ float value(uint32_t bits) {
    if constexpr (TYPE == ATSPEED_F32) return __uint_as_float(bits);
    else return unpack2(bits, TYPE == ATSPEED_F16).x;
  }
};
// A thread's logits of a tile, as they are in memory; which of them it is by constants alone.
template <int TYPE>
struct Tile {
  uint32_t w[kVec][4];
  __device__ __forceinline__ float at(int v, int j) const {
    if constexpr (TYPE == ATSPEED_F32) return __uint_as_float(w[v][j]);
    else if constexpr (TYPE == ATSPEED_BF16) return __uint_as_float(j & 1 ? w[v][j / 2] & 0xffff0000u : w[v][j / 2] << 16);
    else return j & 1 ? unpack2(w[v][j / 2], true).y : unpack2(w[v][j / 2], true).x;
  }
  __device__ __forceinline__ void set(int v, int j, uint32_t bits) {
    if constexpr (TYPE == ATSPEED_F32) w[v][j] = bits;
    else w[v][j / 2] = j & 1 ? (w[v][j / 2] & 0xffffu) | bits << 16 : (w[v][j / 2] & 0xffff0000u) | bits;
  }
};

// The largest t with at least `want` of n keys in shared memory at or above it, or a smaller one with at most `most` there; 0
// where fewer than `want` are above kNone.  A warp.
__device__ __forceinline__ uint32_t threshold_of(const uint32_t* keys, int n, int want, int most) {
  const int lane = threadIdx.x & 31;
  uint32_t lo = 0xffffffffu, hi = 0;
  int valid = 0;
#pragma unroll 4
  for (int i = lane; i < n; i += 32) {
    const uint32_t k = keys[i];
    if (k > kNone) lo = min(lo, k), hi = max(hi, k), ++valid;
  }
  valid = __reduce_add_sync(0xffffffffu, valid);
  if (valid < want) return 0;
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (valid <= most) return lo;
  while (lo < hi) {   // at least `want` at lo, fewer above hi
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    int c = 0;
#pragma unroll 8
    for (int i = lane; i < n; i += 32) c += keys[i] >= mid;
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
  uint32_t group[kVec * kThreads];
  uint32_t from;
  int n;             // candidates in the list, once they are known
  int more[3];       // what tiles add to it, one after the other
  int count[kWarps];
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
__device__ __noinline__ uint32_t cut_list(Shared& sh, int W) {
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

// The W best of a tile's tokens [t0, end), where more than the list holds are at or above `from`, exactly: into the list behind its `had`
// candidates (equal ones in the tokens' order).  Reads the tile again.  Every thread of the CTA; returns what the list then holds.
template <int TYPE>
__device__ __noinline__ int put_exactly(const SelectArgs& a, const char* in, const uint32_t* allowed, int t0, int end, uint32_t from, int had,
                                        Shared& sh) {
  const int tid = threadIdx.x;
  const auto key = [&](int t) {
    if (t >= end || (allowed && !(__ldg(allowed + (t >> 5)) >> (t & 31) & 1))) return 0u;
    using Bits = std::conditional_t<In<TYPE>::SIZE == 4, uint32_t, uint16_t>;
    const float y = In<TYPE>::value(__ldg(reinterpret_cast<const Bits*>(in) + t));
    const uint32_t k = y == y ? key_of(fminf(y, In<TYPE>::value(In<TYPE>::MOST))) : 0u;
    return k >= from ? k : 0u;
  };
  uint32_t lo = from, hi = 0xffffffffu;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    int c = 0;
    for (int t = t0 + tid; t < t0 + In<TYPE>::TILE; t += kThreads) c += key(t) >= mid;
    if (block_count(c, sh) >= a.W) lo = mid;
    else hi = mid - 1;
  }
  int above = 0;
  for (int t = t0 + tid; t < t0 + In<TYPE>::TILE; t += kThreads) above += key(t) > lo;
  above = block_count(above, sh);
  if (tid == 0) sh.n = had;
  __syncthreads();
  int at = had + above, room = a.W - above;   // of the equal ones (at least one)
  for (int t1 = t0; t1 < t0 + In<TYPE>::TILE; t1 += kThreads) {
    const uint32_t k = key(t1 + tid);
    const unsigned same = __ballot_sync(0xffffffffu, k == lo);
    const int all = room > 0 ? block_count((tid & 31) == 0 ? __popc(same) : 0, sh) : 0;   // (sh.count: the warps')
    int place = -1;
    if (k > lo) {
      place = atomicAdd(&sh.n, 1);
    } else if (k == lo) {
      int nth = __popc(same & ((1u << (tid & 31)) - 1u));
      for (int w = 0; w < tid >> 5; ++w) nth += sh.count[w];
      if (nth < room) place = at + nth;
    }
    if (place >= 0) {
      sh.key[place] = k;
      sh.tok[place] = t1 + tid;
    }
    at += min(room, all);
    room -= min(room, all);
  }
  __syncthreads();
  return at;
}

// ALIGNED: every row begins at a multiple of 16 bytes.
template <int TYPE, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, ALIGNED ? 4 : 3) beam_pieces_kernel(const __grid_constant__ SelectArgs a) {
  constexpr int N = In<TYPE>::N, SIZE = In<TYPE>::SIZE, TILE = In<TYPE>::TILE;
  __shared__ Shared sh;
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch_dependents();
  const int begin = piece * a.span, end = min(a.V, begin + a.span);
  const char* in = static_cast<const char*>(a.logits) + (long long)row * a.ld * SIZE;
  const unsigned lead = ALIGNED ? 0u : (unsigned)(reinterpret_cast<uintptr_t>(in) & 15);   // bytes that the row begins behind a 16-byte word
  const auto token = [&](int t0, int v) { return t0 + (v * kThreads + tid) * N; };   // the first of a vector
  // A thread's logits of a tile, wherever the row begins: the 16-byte words that they lie in, shifted.  At a row's ends one by one.
  const auto load = [&](int t0, Tile<TYPE>& x) {
    if (ALIGNED && t0 + TILE <= end) {
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        const uint4 p = __ldcs(reinterpret_cast<const uint4*>(in + (long long)token(t0, v) * SIZE));
        x.w[v][0] = p.x, x.w[v][1] = p.y, x.w[v][2] = p.z, x.w[v][3] = p.w;
      }
      return;
    }
    if (!ALIGNED && t0 > 0 && t0 + TILE + N <= end) {
      uint4 p[kVec], q[kVec];
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        const uint4* at = reinterpret_cast<const uint4*>(in + (long long)token(t0, v) * SIZE - lead);
        p[v] = __ldg(at);
        q[v] = __ldg(at + 1);   // (lead 0: not needed; the other words of a line that is read anyway)
      }
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        uint32_t y[8] = {p[v].x, p[v].y, p[v].z, p[v].w, q[v].x, q[v].y, q[v].z, q[v].w};
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
#pragma unroll
        for (int j = 0; j < 4; ++j) x.w[v][j] = y[j];
      }
      return;
    }
#pragma unroll
    for (int v = 0; v < kVec; ++v) {
      const int t = token(t0, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (SIZE == 4) {
          x.w[v][j] = t + j < end ? __ldg(reinterpret_cast<const uint32_t*>(in) + t + j) : In<TYPE>::NONE;
        } else {
          const uint16_t* h = reinterpret_cast<const uint16_t*>(in);
          const uint32_t lo = t + 2 * j < end ? __ldg(h + t + 2 * j) : In<TYPE>::NONE;
          const uint32_t hi = t + 2 * j + 1 < end ? __ldg(h + t + 2 * j + 1) : In<TYPE>::NONE;
          x.w[v][j] = lo | hi << 16;
        }
      }
    }
  };
  const int cu0 = __ldg(a.cu), cu1 = __ldg(a.cu + a.n_req);
  if (row < cu0 || row >= cu1 || (a.final && __ldg(a.final + row) >= 0)) return;   // (the other kernel knows as much)
  const int st = a.state ? __ldg(a.state + row) : -1;
  const uint32_t* allowed = st >= 0 && st < a.n_states ? a.grammar + st * a.grammar_stride : nullptr;
  const bool nothing = st >= a.n_states && a.state;
  Tile<TYPE> x;
  load(begin, x);
  if (tid < 3) sh.more[tid] = 0;
  float m = -INFINITY, s = 0.f;   // the thread's maximum and sum
  uint32_t floor = kNone;         // only what is above it is a candidate
  bool open = true;               // .. and fewer than W are known at or above a bound
  int n = 0, again = 0;           // candidates in the list; how many there may be before the bound is looked for anew
  __syncthreads();
  for (int t0 = begin, turn = 0; t0 < end; t0 += TILE, turn = turn == 2 ? 0 : turn + 1) {
    const auto each = [&](auto&& f) {
#pragma unroll
      for (int v = 0; v < kVec; ++v)
#pragma unroll
        for (int j = 0; j < N; ++j) f(v, j);
    };
    uint32_t ok = 0xffffffffu;   // bit v N + j: that token is allowed
    if (allowed) {
      ok = 0;
#pragma unroll
      for (int v = 0; v < kVec; ++v) {   // (a vector's bits lie in one word)
        const int t = token(t0, v);
        if (t < end) ok |= (__ldg(allowed + (t >> 5)) >> (t & 31) & ((1u << N) - 1)) << v * N;
      }
    } else if (nothing) {
      ok = 0;
    }
    const bool hidden = allowed || nothing;
    const auto hide = [&] {
      each([&](int v, int j) {
        if (!(ok >> (v * N + j) & 1)) x.set(v, j, In<TYPE>::NONE);
      });
    };
    float vm[kVec], top;   // of the vectors, of all (a NaN is passed over)
    const auto tops = [&] {
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        vm[v] = fmaxf(x.at(v, 0), x.at(v, 1));
#pragma unroll
        for (int j = 2; j < N; ++j) vm[v] = fmaxf(vm[v], x.at(v, j));
        vm[v] = fmaxf(vm[v], -INFINITY);
      }
      top = vm[0];
#pragma unroll
      for (int v = 1; v < kVec; ++v) top = fmaxf(top, vm[v]);
    };
    if (hidden && !a.full) hide();
    tops();
    float sum = 0.f, M = fmaxf(m, top);
    if (M > -INFINITY) {
      if (fabsf(M) < kFar) {
        const float u = unit_of(M);
        float more = 0.f;
        each([&](int v, int j) { (j & 1 ? more : sum) += exp2_approx(fmaf(x.at(v, j), kLog2e, -u)); });
        sum += more;
      } else {
        sum = NAN;
      }
      if (sum != sum) {   // a NaN (it counts as -infinity), an infinity (as the type's largest), logits far out
        each([&](int v, int j) {
          const float y = x.at(v, j);
          if (y != y) x.set(v, j, In<TYPE>::NONE);
          else if (y == INFINITY) x.set(v, j, In<TYPE>::MOST);
        });
        tops();
        M = fmaxf(m, top);
        sum = 0.f;
        const bool near = fabsf(M) < kFar;
        const float u = unit_of(M);
        if (M > -INFINITY) each([&](int v, int j) { sum += exp2_approx(near ? fmaf(x.at(v, j), kLog2e, -u) : (x.at(v, j) - M) * kLog2e); });
      }
      if (M > m) {
        s = m > -INFINITY ? s * rescale(m, M) : 0.f;
        m = M;
      }
    }
    s += sum;
    if (hidden && a.full) {
      hide();
      tops();
    }
    uint32_t from = floor + 1, bound = 0;
    if (open) {   // from the W-th of the groups' maxima on
      int groups = kThreads;
      if (a.W <= 32) {
        sh.group[tid] = key_of(top);
      } else if (a.W <= 128) {
        sh.group[tid] = key_of(fmaxf(vm[0], vm[1]));
        sh.group[kThreads + tid] = key_of(fmaxf(vm[2], vm[3]));
        groups = 2 * kThreads;
      } else {
#pragma unroll
        for (int v = 0; v < kVec; ++v) sh.group[v * kThreads + tid] = key_of(vm[v]);
        groups = kVec * kThreads;
      }
      __syncthreads();
      if (warp == 0) {
        const uint32_t t = threshold_of(sh.group, groups, a.W, a.W + a.W / 4);
        if (lane == 0) sh.from = t;
      }
      __syncthreads();
      bound = sh.from;
      from = max(from, bound);
    }
    const float least = value_of(from);
    if (top >= least)
      each([&](int v, int j) {
        const float y = x.at(v, j);
        if (y >= least) {
          const int at = n + atomicAdd(&sh.more[turn], 1);
          if (at < kList) {
            sh.key[at] = key_of(y);
            sh.tok[at] = token(t0, v) + j;
          }
        }
      });
    if (tid == 0) sh.more[turn == 2 ? 0 : turn + 1] = 0;   // (last read two barriers ago)
    __syncthreads();
    const int had = n;
    n += sh.more[turn];
    if (n > kList) n = put_exactly<TYPE>(a, in, allowed, t0, end, from, had, sh);
    if (t0 + TILE < end) load(t0 + TILE, x);
    if (bound) {   // (W of the tile's are at `from` or above: a later token there comes after them)
      open = false;
      floor = from;
      again = n + a.W / 2;
    }
    if (n > kList / 2) {
      if (tid == 0) sh.n = n;
      open = false;
      floor = max(floor, cut_list(sh, a.W));
      n = a.W;
      again = n + a.W / 2;
    } else if (!open && n > again && t0 + TILE < end) {   // a better bound: the W-th (or so) of the list
      if (warp == 0) {
        const uint32_t t = threshold_of(sh.key, n, a.W, a.W + a.W / 4);
        if (lane == 0) sh.from = t;
      }
      __syncthreads();
      floor = max(floor, sh.from);
      again = n + a.W / 2;
    }
  }
  // hands on the list, or what is at or above a bound that leaves few enough
  const long long at = (long long)row * a.pieces + piece;
  uint32_t from = 0;
  if (n > a.cap) {
    if (warp == 0) {
      const uint32_t t = threshold_of(sh.key, n, a.W, a.cap);
      int c = 0;
      for (int i = lane; i < n; i += 32) c += sh.key[i] >= t;
      c = __reduce_add_sync(0xffffffffu, c);
      if (lane == 0) {
        sh.from = t;
        sh.n = c;
      }
    }
    __syncthreads();
    from = sh.from;
    if (sh.n > a.cap) {   // (equal ones)
      __syncthreads();
      if (tid == 0) sh.n = n;
      cut_list(sh, a.W);
      n = a.W;
      from = 0;
    }
    __syncthreads();
  }
  if (tid == 0) sh.n = 0;
  // the piece's sum, in one order
  float M = warp_max(m);
  if (lane == 0) sh.m[warp] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sh.m[w]);
  const float sum = warp_sum(m > -INFINITY ? s * rescale(m, M) : 0.f);
  if (lane == 0) sh.s[warp] = sum;
  for (int i = tid; i < n; i += kThreads)
    if (sh.key[i] >= from) a.cand[at * a.cap + atomicAdd(&sh.n, 1)] = make_uint2(__float_as_uint(value_of(sh.key[i])), (uint32_t)sh.tok[i]);
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
  float cum, off32, more32;
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
  const auto row_at = [&](int r) -> Row& { return r - r0 < kRows ? sh.row[r - r0] : a.rows[r]; };
  // A row's maximum and sum from its pieces: many pieces by a warp, few by a thread; then its logarithm.
  // (Sums as multiples of 2^-32, whole numbers: a row's is at least 0.7 and at most 1.5 times its length.)
  const auto whole = [&](float s) { return (unsigned long long)(s * 0x1p32f); };
  const auto set_row = [&](int r, float M, unsigned long long s) {
    Row w = {0.0, 0.0, a.score ? __ldg(a.score + r) : 0.f, 0.f, 0.f, -1};
    const double l = log((double)s * 0x1p-32);
    if (fabsf(M) < kFar) w.off = (double)unit_of(M) * kLn2 + l - (double)M * kEta;
    else w.off = (double)M, w.more = l;
    w.off32 = (float)w.off, w.more32 = (float)w.more;
    row_at(r) = w;
  };
  const auto final_of = [&](int r) { return a.final ? __ldg(a.final + r) : -1; };
  const auto set_final = [&](int r, int f) { row_at(r) = {0.0, 0.0, a.score ? __ldg(a.score + r) : 0.f, 0.f, 0.f, f}; };
  if (a.pieces <= 2) {
    for (int r = r0 + tid; r < r1; r += kRankThreads) {
      const int f = final_of(r);
      if (f >= 0) {
        set_final(r, f);
        continue;
      }
      const Header* h = a.head + (long long)r * a.pieces;
      const float m0 = h[0].m, s0 = h[0].s, m1 = a.pieces > 1 ? h[1].m : -INFINITY, s1 = a.pieces > 1 ? h[1].s : 0.f;
      const float M = fmaxf(m0, m1);
      set_row(r, M, M > -INFINITY ? whole(s0 * rescale(m0, M)) + whole(s1 * rescale(m1, M)) : 0ull);
    }
  } else {
    for (int base = r0; base < r1; base += kRankThreads) {   // (a thousand rows at a time, whose sums wait in the list's place)
      const int last = min(r1, base + kRankThreads);
      for (int r = base + warp; r < last; r += kRankThreads / 32) {
        const Header* h = a.head + (long long)r * a.pieces;
        const bool live = final_of(r) < 0;
        float M = -INFINITY;
        for (int p = lane; live && p < a.pieces; p += 32) M = fmaxf(M, h[p].m);
        M = warp_max(M);
        unsigned long long s = 0;
        for (int p = lane; live && p < a.pieces; p += 32)
          if (h[p].m > -INFINITY) s += whole(h[p].s * rescale(h[p].m, M));
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) {
          sh.group[r - base] = __float_as_uint(M);
          sh.score[r - base] = s;
        }
      }
      __syncthreads();
      if (base + tid < last) {
        const int r = base + tid, f = final_of(r);
        if (f >= 0) set_final(r, f);
        else set_row(r, __uint_as_float(sh.group[tid]), sh.score[tid]);
      }
      __syncthreads();
    }
  }
  __syncthreads();
  // Candidates: a thread has place `at` of list my_list and of every lists_at_once-th list from there.
  const int lists_at_once = kRankThreads / a.cap, at = tid % a.cap, my_list = tid / a.cap;
  const auto fetch = [&](int l, uint2& c, int& n) {
    const long long h = (long long)r0 * a.pieces + l;
    c = a.cand[h * a.cap + at];
    n = a.head[h].n;
  };
  // Its score in 32 bits, and how far that may be off (four roundings); false: there is none
  const auto look = [&](int l, uint2& c, int n, float& y, float& e) {
    const Row& w = row_at(r0 + l / a.pieces);
    if (w.final >= 0) {
      c = make_uint2(0u, (uint32_t)w.final);
      y = w.cum, e = 0.f;
      return at == 0 && l % a.pieces == 0;
    }
    const float x = __uint_as_float(c.x);
    y = w.cum + ((x - w.off32) - w.more32);
    e = 0x1p-21f * (fabsf(w.cum) + fabsf(x) + fabsf(w.off32) + fabsf(w.more32));
    return at < n;
  };
  // what is below `from` is not among the W best: the W-th of the threads' best (some of them have W candidates, or they are few)
  constexpr int kHold = 4;
  const bool hold = lists <= kHold * lists_at_once;
  uint2 c[kHold];
  int cn[kHold];
  float g = -INFINITY;
  for (int l0 = 0; l0 < lists; l0 += kHold * lists_at_once) {
#pragma unroll
    for (int q = 0; q < kHold; ++q) {
      cn[q] = 0;
      const int l = l0 + q * lists_at_once + my_list;
      if (l < lists) fetch(l, c[q], cn[q]);
    }
#pragma unroll
    for (int q = 0; q < kHold; ++q) {
      const int l = l0 + q * lists_at_once + my_list;
      float y, e;
      if (l < lists && look(l, c[q], cn[q], y, e)) g = fmaxf(g, y - e);   // (not a NaN)
    }
  }
  sh.group[tid] = key_of(g);
  __syncthreads();
  if (warp == 0) {
    const uint32_t t = threshold_of(sh.group, kRankThreads, a.W, a.W + a.W / 4);
    if (lane == 0) sh.from = t;
  }
  __syncthreads();
  float from = sh.from ? value_of(sh.from) : -INFINITY;
  const auto put = [&](int l, uint2 c, int n) {
    float y, e;
    if (!look(l, c, n, y, e) || y + e < from) return;
    const int r = r0 + l / a.pieces;
    const Row& w = row_at(r);
    const float x = __uint_as_float(c.x);
    const double z = w.final >= 0 ? (double)w.cum : (double)w.cum + (((double)x - w.off) - w.more);
    if (!((float)z > -INFINITY)) return;
    const int to = atomicAdd(&sh.n, 1);
    sh.score[to] = key_of(z + 0.0);   // (-0: 0)
    sh.rest[to] = (unsigned long long)(~(uint32_t)r) << 32 | key_of(x);
    sh.tok[to] = c.y;
  };
#pragma unroll 1
  for (int l0 = 0, q = 0; l0 < lists; l0 += lists_at_once, ++q) {
    const int l = l0 + my_list;
    if (l < lists) {
      uint2 x = q == 0 ? c[0] : q == 1 ? c[1] : q == 2 ? c[2] : c[3];
      int n = q == 0 ? cn[0] : q == 1 ? cn[1] : q == 2 ? cn[2] : cn[3];
      if (!hold) fetch(l, x, n);
      put(l, x, n);
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

constexpr int kTile = In<ATSPEED_F32>::TILE;
// Pieces of a row: enough CTAs for every SM to have four, none shorter than a tile.
int pieces_of(int R, int V) {
  const long long tiles = (V + kTile - 1LL) / kTile;   // (of the smaller tile)
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
  const bool aligned = aligned16(d_logits) && ld * dtype_size(type) % 16 == 0;
  const auto go = [&](auto kernel) { kernel<<<grid, kThreads, 0, (cudaStream_t)stream>>>(a); };
  if (type == ATSPEED_F32) aligned ? go(beam_pieces_kernel<ATSPEED_F32, true>) : go(beam_pieces_kernel<ATSPEED_F32, false>);
  else if (type == ATSPEED_BF16) aligned ? go(beam_pieces_kernel<ATSPEED_BF16, true>) : go(beam_pieces_kernel<ATSPEED_BF16, false>);
  else aligned ? go(beam_pieces_kernel<ATSPEED_F16, true>) : go(beam_pieces_kernel<ATSPEED_F16, false>);
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
