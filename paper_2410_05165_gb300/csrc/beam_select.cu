// Beam search's selection over beams and vocabulary (atspeed_op_beam_select).
//   score(r, v) = cum_r + ((x_rv - m_r) - log s_r),  m_r = max x_r,  s_r = sum_v exp(x_rv - m_r);  the best W of a request's rows
// Bound: HBM (each logit read once).  3840 rows of 33024 (32 bits, W = 80) take 99 us, 5.1 TB/s: 75 of them the logits alone (a copy's rate), 3
// the bounds, 10 the second reads, 10 the ranking.  738 rows of 100003 (bf16, at odd addresses, W = 32) 38 us, 3.9 TB/s, where
// unpacking and exponentials take as long as the bytes.  Ten rows of 33024 11 us: latency, half of it the ranking's.
//
// Two launches.  The first reads the logits, a CTA a piece of a row: the piece's maximum, its sum of exponentials and the
// candidates among its logits, which are at least its W best (within a row the order is the logits').  The second, a CTA a
// request, makes log s_r of the pieces, looks at the candidates in 32 bits and ranks those that may be among the best.
//
// Candidates of a piece: its tokens form groups (128 to 512, each some of a thread's, strided over the whole piece) whose maxima stay in
// registers while the logits stream by.  W of these maxima, so W logits, are at or above the W-th largest of them: the groups that
// reach that bound, little more than W of them, are read again for what is at or above it: in the one tile that holds the
// maximum, or in all if the next best reaches the bound too.  (Logits held against a bound as they come: 290 us for the 3840 rows; every
// tile of those groups read again: 116.)  Of more than are handed on, a bound among them leaves fewer; where the logits are equal or
// more than a list holds reach the bound (a mask of the type's lowest value), the W best are searched exactly.
//
// Logits come through a ring of asynchronous copies, two tiles ahead: 64 to 80 KB an SM under way.  CTAs of 128 threads, so that few of an
// SM's are at their bounds, which take a fifth of a row's time, while the others read.  Sums of a row do not depend on where the
// row begins in memory, so that rows with the same logits have the same bits.
#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32, kCtas = 5;   // (CTAs an SM)
constexpr int kVec = 4;                     // 16-byte vectors of a thread in a tile
constexpr int kList = 1024;                 // candidates that a piece's list holds
constexpr int kGroups = kThreads * kVec;
constexpr int kMaxWidth = 256;
constexpr uint32_t kNone = 0x007fffffu;     // the key of -infinity

struct Header {   // of a piece
  float m, s;
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
  uint32_t per_piece;   // 2^32 / pieces, rounded up
  int *token, *parent;
  float* out_score;
  Header* head;
  uint2* cand;   // (logit, token)
  struct Row* rows;   // [R]
  struct Quick* quick;
};

// Order-preserving maps to whole numbers.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);   // (-0: 0)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// Sums in two 32-bit parts, the larger rounded to nearest (64-bit arithmetic has a hundred clocks of latency here: with it the ranking of
// ten beams took 2 us more).
struct Two {
  float hi, lo;
};
__device__ __forceinline__ Two two_sum(float a, float b) {   // a + b exactly (Knuth)
  const float s = a + b, c = s - a;
  return {s, (a - (s - c)) + (b - c)};
}
__device__ __forceinline__ Two add_low(Two a, float lo) {   // |lo| << |a.hi|; what is not finite has no lower part
  if (!(fabsf(a.hi) < INFINITY)) return {a.hi, 0.f};
  lo += a.lo;
  const float hi = a.hi + lo;
  return {hi, lo - (hi - a.hi)};
}
__device__ __forceinline__ unsigned long long key_of(Two a) { return (unsigned long long)key_of(a.hi) << 32 | key_of(a.lo); }

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
// Logit j of a vector; of a thread's logits of a tile, as they are in memory (which of them it is by constants alone).
template <int TYPE>
__device__ __forceinline__ float vector_at(const uint32_t (&w)[4], int j) {
  if constexpr (TYPE == ATSPEED_F32) return __uint_as_float(w[j]);
  else if constexpr (TYPE == ATSPEED_BF16) return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
  else return j & 1 ? unpack2(w[j / 2], true).y : unpack2(w[j / 2], true).x;
}
template <int TYPE>
struct Tile {
  uint32_t w[kVec][4];
  __device__ __forceinline__ float at(int v, int j) const { return vector_at<TYPE>(w[v], j); }
  __device__ __forceinline__ void set(int v, int j, uint32_t bits) {
    if constexpr (TYPE == ATSPEED_F32) w[v][j] = bits;
    else w[v][j / 2] = j & 1 ? (w[v][j / 2] & 0xffffu) | bits << 16 : (w[v][j / 2] & 0xffff0000u) | bits;
  }
};

// The largest t with at least `want` of the CTA's keys (E a thread) at or above it, or a smaller one with at most `most` there; 0
// where fewer than `want` are above kNone.  Every thread of the CTA; scratch: 3 words a warp.  (The barriers count: by one warp, with
// the keys in shared memory, it took twice as long.)
template <int E, int WARPS>
__device__ __forceinline__ uint32_t threshold_of(const uint32_t (&k)[E], int want, int most, uint32_t* scratch) {
  uint32_t lo = 0xffffffffu, hi = 0, valid = 0;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (k[e] > kNone) lo = min(lo, k[e]), hi = max(hi, k[e]), ++valid;
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  valid = __reduce_add_sync(0xffffffffu, valid);
  const int lane = threadIdx.x & 31;
  if (lane == 0) {
    uint32_t* at = scratch + threadIdx.x / 32;
    at[0] = lo, at[WARPS] = hi, at[2 * WARPS] = valid;
  }
  __syncthreads();
  const bool have = lane < WARPS;
  lo = __reduce_min_sync(0xffffffffu, have ? scratch[lane] : 0xffffffffu);
  hi = __reduce_max_sync(0xffffffffu, have ? scratch[WARPS + lane] : 0u);
  valid = __reduce_add_sync(0xffffffffu, have ? scratch[2 * WARPS + lane] : 0u);
  if ((int)valid < want) return 0;
  if ((int)valid <= most) return lo;
  while (lo < hi) {   // at least `want` at lo, fewer above hi
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    int c = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) c += __syncthreads_count(k[e] >= mid);
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
  uint32_t scratch[3 * kWarps];
  int read[kGroups];         // vectors to be read again: from the front by their first tokens, from the back in every tile
  int n, n_reads, count[kWarps], same[kWarps];   // n_reads: those at the front, and 65536 times those at the back
  float m[kWarps], s[kWarps];
};

// A sum of exponentials below a maximum m: for |m| < kFar in units of the whole power of two 2^unit_of(m), its terms 2^(x l - unit)
// by one multiply-add (l = log2 e in 32 bits), so that another maximum rescales it exactly, whatever their order; from
// kFar on, where x l has no bits left for that, in units of e^m.
// e^x as 2^(x l) is off by a factor e^(x kEta), which the scores take back for the row's maximum.
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.69314718055994530942;
constexpr float kLn2Hi = (float)kLn2, kLn2Lo = (float)(kLn2 - (double)kLn2Hi), kEta = (float)((double)kLog2e * kLn2 - 1.0);
constexpr float kFar = 0x1p20f;

__device__ __forceinline__ float unit_of(float m) { return rintf(m * kLog2e); }
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The even and the odd ones of a thread's 2^(x l + c), i < kVec N, added up (two at a time: an instruction less for each).
template <int COUNT, class X>
__device__ __forceinline__ void sum_exp2(X&& x, float c, float& even, float& odd) {
  unsigned long long l, add, sum = 0, y;
  asm("mov.b64 %0, {%1, %1};" : "=l"(l) : "f"(kLog2e));
  asm("mov.b64 %0, {%1, %1};" : "=l"(add) : "f"(c));
#pragma unroll
  for (int i = 0; i < COUNT; i += 2) {
    float a, b;
    asm("{\n .reg .b64 p;\n mov.b64 p, {%1, %2};\n fma.rn.f32x2 %0, p, %3, %4;\n}" : "=l"(y) : "f"(x(i)), "f"(x(i + 1)), "l"(l), "l"(add));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(y));
    a = exp2_approx(a), b = exp2_approx(b);
    asm("{\n .reg .b64 p;\n mov.b64 p, {%1, %2};\n add.rn.f32x2 %0, %0, p;\n}" : "+l"(sum) : "f"(a), "f"(b));
  }
  asm("mov.b64 {%0, %1}, %2;" : "=f"(even), "=f"(odd) : "l"(sum));
}
// What a sum below m is worth below M >= m.
__device__ __forceinline__ float rescale(float m, float M) {
  if (m == M) return 1.f;
  const bool near = fabsf(m) < kFar, NEAR = fabsf(M) < kFar;
  return exp2_approx(near ? NEAR ? unit_of(m) - unit_of(M) : fmaf(-M, kLog2e, unit_of(m))
                          : NEAR ? fmaf(m, kLog2e, -unit_of(M)) : (m - M) * kLog2e);
}

// A token's key, 0 if it is not a candidate at or above `from`.
template <int TYPE>
__device__ __forceinline__ uint32_t key_at(const char* in, const uint32_t* allowed, int t, uint32_t from) {
  if (allowed && !(__ldg(allowed + (t >> 5)) >> (t & 31) & 1)) return 0u;
  using Bits = std::conditional_t<In<TYPE>::SIZE == 4, uint32_t, uint16_t>;
  const float y = In<TYPE>::value(__ldg(reinterpret_cast<const Bits*>(in) + t));
  const uint32_t k = y == y ? key_of(fminf(y, In<TYPE>::value(In<TYPE>::MOST))) : 0u;   // (NaN: -infinity)
  return k >= from ? k : 0u;
}

// The W best of the tokens [begin, end), of which more than W are at or above `from`, exactly (equal ones in the tokens' order), into the
// list.  Every thread of the CTA; a warp has a share of the tokens, in order.  A pass over them halves the keys that the W-th best may have
// and goes on to the next one that there is, so that few different logits need few passes: 3840 rows of 33024 take 867 us where they are
// whole numbers in bf16 (6015 with the halving alone; 75 where no row needs this), 1121 where all are equal in 32 bits (3083 with barriers
// for every 128 tokens and the ranking by a thousand threads at a time; 100 where no row needs this).  `most`: no key is above it.
template <int TYPE>
__device__ __noinline__ void put_exactly(const char* in, const uint32_t* allowed, int begin, int end, uint32_t from, uint32_t most, int W, Shared& sh) {
  constexpr int kAtOnce = 8;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int share = (end - begin + 32 * kWarps - 1) / (32 * kWarps) * 32, t0 = begin + warp * share, t1 = min(end, t0 + share);
  const auto each = [&](uint32_t least, auto&& go) {   // go(token, key at or above `least` or 0), 32 tokens after 32
    for (int t = t0; t < t1; t += 32 * kAtOnce) {
      uint32_t k[kAtOnce];
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) k[q] = t + 32 * q + lane < t1 ? key_at<TYPE>(in, allowed, t + 32 * q + lane, least) : 0u;
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) go(t + 32 * q + lane, k[q]);
    }
  };
  int above, before, same;     // of all tokens above lo; at lo, of the warps before this one and of this one
  uint32_t lo = from, hi = most;   // at least W are at or above lo, fewer above hi
  while (true) {
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    int up = 0, at = 0, mids = 0;    // above lo, at it, at or above mid
    uint32_t next = ~0u, mid_next = ~0u;   // the smallest of them
    each(lo, [&](int, uint32_t k) {
      at += k == lo;
      if (k > lo) ++up, next = min(next, k);
      if (k >= mid) ++mids, mid_next = min(mid_next, k);
    });
    up = __reduce_add_sync(0xffffffffu, up), same = __reduce_add_sync(0xffffffffu, at), mids = __reduce_add_sync(0xffffffffu, mids);
    next = __reduce_min_sync(0xffffffffu, next), mid_next = __reduce_min_sync(0xffffffffu, mid_next);
    __syncthreads();
    if (lane == 0) {
      sh.count[warp] = up, sh.same[warp] = same;
      sh.scratch[warp] = (uint32_t)mids, sh.scratch[kWarps + warp] = next, sh.scratch[2 * kWarps + warp] = mid_next;
    }
    __syncthreads();
    above = before = mids = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      above += sh.count[w], before += w < warp ? sh.same[w] : 0;
      mids += (int)sh.scratch[w], next = min(next, sh.scratch[kWarps + w]), mid_next = min(mid_next, sh.scratch[2 * kWarps + w]);
    }
    if (above < W) break;
    if (mids >= W) lo = mid_next;
    else lo = next, hi = mid - 1;
  }
  if (tid == 0) sh.n = 0;
  __syncthreads();
  int at = above + before;
  each(lo, [&](int t, uint32_t k) {
    const unsigned equal = __ballot_sync(0xffffffffu, k == lo);
    int place = k > lo ? atomicAdd(&sh.n, 1) : k == lo ? at + __popc(equal & ((1u << lane) - 1u)) : W;
    at += __popc(equal);
    if (place < W) {
      sh.key[place] = k;
      sh.tok[place] = t;
    }
  });
  __syncthreads();
  if (tid == 0) sh.n = W;
  __syncthreads();
}

// A tile's 16-byte words on their way through shared memory, a warp's 32 of a vector in a row, and the one behind them.
constexpr int kStages = 3;   // (two tiles under way)
struct Stage {
  uint4 word[kWarps][kVec][33];
};
union PieceShared {
  Stage ring[kStages];   // while the logits stream by
  Shared sh;             // then
};

// The first `bytes` of 16 from device to shared memory, zeros behind them.
__device__ __forceinline__ void copy16(void* to, const void* from, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory");
}

// ALIGNED: every row begins at a multiple of 16 bytes.
template <int TYPE, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, kCtas) beam_pieces_kernel(const __grid_constant__ SelectArgs a) {
  constexpr int N = In<TYPE>::N, SIZE = In<TYPE>::SIZE, TILE = In<TYPE>::TILE;
  extern __shared__ __align__(16) unsigned char raw[];
  PieceShared& shared = *reinterpret_cast<PieceShared*>(raw);
  Shared& sh = shared.sh;
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch_dependents();
  const int begin = piece * a.span, end = min(a.V, begin + a.span);
  const char* in = static_cast<const char*>(a.logits) + (long long)row * a.ld * SIZE;
  const unsigned lead = ALIGNED ? 0u : (unsigned)(reinterpret_cast<uintptr_t>(in) & 15);   // bytes that the row begins behind a 16-byte word
  const auto token = [&](int t0, int v) { return t0 + (v * kThreads + tid) * N; };   // the first of a vector
  // (A word that the row begins in holds bytes of it, so it may be read; behind the piece's end nothing is.)
  const auto fetch = [&](int t0, int stage) {
    if (t0 < end) {
      const char* from = in - lead + (long long)token(t0, 0) * SIZE;
      auto& to = shared.ring[stage].word[warp];
      if (t0 + TILE + N <= end) {
#pragma unroll
        for (int v = 0; v < kVec; ++v) copy16(&to[v][lane], from + v * kThreads * 16, 16);
        if (!ALIGNED && lane < kVec) copy16(&to[lane][32], from + (lane * kThreads + 32 - lane) * 16, 16);
      } else {
        const char* stop = in + (long long)end * SIZE;
        const auto some = [&](uint4* to, const char* from) {
          const long long left = stop - from;
          copy16(to, left > 0 ? from : in - lead, left > 0 ? (int)min(16ll, left) : 0);   // (a multiple of 16, if nothing is read there too)
        };
#pragma unroll
        for (int v = 0; v < kVec; ++v) some(&to[v][lane], from + v * kThreads * 16);
        if (!ALIGNED && lane < kVec) some(&to[lane][32], from + (lane * kThreads + 32 - lane) * 16);
      }
    }
    copies_done();
  };
  // the 16 bytes that begin `lead` bytes into p: words from the (lead / 4)-th on, each with the half that follows it
  const auto shift_by = [&](auto words, const uint4& p, const uint4& q, uint32_t (&w)[4]) {
    const uint32_t y[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = SIZE == 2 ? __funnelshift_r(y[j + words], y[j + words + 1], lead * 8) : y[j + words];   // (its low 5 bits: 0 or 16)
  };
  const auto with_words = [&](auto&& f) {
    switch (lead / 4) {
      case 0: f(std::integral_constant<int, 0>()); break;
      case 1: f(std::integral_constant<int, 1>()); break;
      case 2: f(std::integral_constant<int, 2>()); break;
      default: f(std::integral_constant<int, 3>());
    }
  };
  // A thread's logits of a tile, wherever the row begins: its words, shifted.
  const auto take = [&](int t0, int stage, Tile<TYPE>& x) {
    const auto& at = shared.ring[stage].word[warp];
    const auto words = [&](auto k) {
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        const uint4 p = at[v][lane];
        if constexpr (ALIGNED) x.w[v][0] = p.x, x.w[v][1] = p.y, x.w[v][2] = p.z, x.w[v][3] = p.w;
        else shift_by(k, p, at[v][lane + 1], x.w[v]);
      }
    };
    if constexpr (ALIGNED) words(0);
    else with_words(words);
    if (t0 + TILE > end) {
#pragma unroll
      for (int v = 0; v < kVec; ++v)
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (token(t0, v) + j >= end) x.set(v, j, In<TYPE>::NONE);
    }
  };
  // The vector of logits from token t on, -infinity behind the end; by the words that it lies in or one by one.
  const auto vector = [&](int t, uint32_t (&w)[4]) {
    if (t + 2 * N <= end) {
      const uint4* at = reinterpret_cast<const uint4*>(in - lead + (long long)t * SIZE);
      const uint4 p = __ldg(at);
      w[0] = p.x, w[1] = p.y, w[2] = p.z, w[3] = p.w;
      if (!ALIGNED && lead) {
        const uint4 q = __ldg(at + 1);
        with_words([&](auto k) { shift_by(k, p, q, w); });
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (SIZE == 4) {
        w[j] = t + j < end ? __ldg(reinterpret_cast<const uint32_t*>(in) + t + j) : In<TYPE>::NONE;
      } else {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(in);
        const uint32_t lo = t + 2 * j < end ? __ldg(h + t + 2 * j) : In<TYPE>::NONE;
        const uint32_t hi = t + 2 * j + 1 < end ? __ldg(h + t + 2 * j + 1) : In<TYPE>::NONE;
        w[j] = lo | hi << 16;
      }
    }
  };
  fetch(begin, 0);
  fetch(begin + TILE, 1);
  const int cu0 = __ldg(a.cu), cu1 = __ldg(a.cu + a.n_req);
  if (row < cu0 || row >= cu1 || (a.final && __ldg(a.final + row) >= 0)) {   // (the other kernel knows as much)
    copies_wait<0>();
    return;
  }
  const int st = a.state ? __ldg(a.state + row) : -1;
  const bool nothing = a.state && st >= a.n_states;
  const uint32_t* allowed = st >= 0 && !nothing ? a.grammar + st * a.grammar_stride : nullptr;
  float m = -INFINITY, s = 0.f;   // the thread's maximum and sum
  float unit = 0.f;               // unit_of(m), a NaN where m is far out
  // .. and of each of its vectors' places: the largest candidate, the tile that it is in, and the largest of the other tiles
  float best[kVec], second[kVec];
  int where[kVec];
#pragma unroll
  for (int v = 0; v < kVec; ++v) best[v] = second[v] = -INFINITY, where[v] = begin;
  Tile<TYPE> x;
  for (int t0 = begin, stage = 0; t0 < end; t0 += TILE, stage = stage == kStages - 1 ? 0 : stage + 1) {
    copies_wait<1>();
    if (!ALIGNED) __syncwarp();
    if (t0 + warp * 32 * N >= end) break;   // (nothing of the last tile is this warp's)
    take(t0, stage, x);
    fetch(t0 + 2 * TILE, stage == 0 ? kStages - 1 : stage - 1);   // (where the tile before this one was)
    const auto each = [&](auto&& f) {
#pragma unroll
      for (int v = 0; v < kVec; ++v)
#pragma unroll
        for (int j = 0; j < N; ++j) f(v, j);
    };
    float vm[kVec], top;   // of the vectors, of all (a NaN is passed over)
    const auto tops = [&] {
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        vm[v] = fmaxf(x.at(v, 0), x.at(v, 1));
#pragma unroll
        for (int j = 2; j < N; ++j) vm[v] = fmaxf(vm[v], x.at(v, j));
      }
      top = vm[0];
#pragma unroll
      for (int v = 1; v < kVec; ++v) top = fmaxf(top, vm[v]);
    };
    uint32_t ok = 0;   // bit v N + j: that token is allowed
    const auto hide = [&] {
      each([&](int v, int j) {
        if (!(ok >> (v * N + j) & 1)) x.set(v, j, In<TYPE>::NONE);
      });
    };
    if (allowed) {
#pragma unroll
      for (int v = 0; v < kVec; ++v) {   // (a vector's bits lie in one word)
        const int t = token(t0, v);
        if (t < end) ok |= (__ldg(allowed + (t >> 5)) >> (t & 31) & ((1u << N) - 1)) << v * N;
      }
      if (!a.full) hide();
    }
    tops();
    float M = fmaxf(m, top);
    const auto unit_at = [&] { return fabsf(M) < kFar ? unit_of(M) : M == -INFINITY ? 0.f : NAN; };   // (nothing yet: any will do)
    float u = unit_at(), sum = 0.f, more = 0.f;
    sum_exp2<kVec * N>([&](int i) { return x.at(i / N, i % N); }, -u, sum, more);
    sum += fmaf(s, exp2_approx(unit - u), more);
    if (sum != sum) {   // a NaN (it counts as -infinity), an infinity (as the type's largest), a maximum far out or of -infinity
      each([&](int v, int j) {
        const float y = x.at(v, j);
        if (y != y) x.set(v, j, In<TYPE>::NONE);
        else if (y == INFINITY) x.set(v, j, In<TYPE>::MOST);
      });
      tops();
      M = fmaxf(m, top);
      u = unit_at();
      sum = 0.f;
      if (M > -INFINITY) {
        each([&](int v, int j) { sum += exp2_approx(u == u ? fmaf(x.at(v, j), kLog2e, -u) : (x.at(v, j) - M) * kLog2e); });
        if (m > -INFINITY) sum += s * rescale(m, M);
      }
    }
    m = M, s = sum, unit = u;
    if (allowed && a.full) {
      hide();
      tops();
    }
#pragma unroll
    for (int v = 0; v < kVec; ++v) {
      second[v] = fmaxf(second[v], fminf(best[v], vm[v]));
      where[v] = vm[v] > best[v] ? t0 : where[v];
      best[v] = fmaxf(best[v], vm[v]);
    }
  }
  __syncthreads();   // (the ring is read)
  // the W-th largest of the groups' maxima, or a smaller value with little more above it: of the threads', for many of their vectors' places
  const float wm = warp_max(m);
  if (lane == 0) sh.m[warp] = wm;
  if (tid == 0) sh.n = sh.n_reads = 0;
  uint32_t from;
  if (a.W <= kThreads / 4) {
    static_assert(kVec == 4, "vectors of a thread");
    const uint32_t k[1] = {key_of(fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3])))};
    from = threshold_of<1, kWarps>(k, a.W, a.W + a.W / 8, sh.scratch);
  } else if (a.W <= 96) {
    const uint32_t k[2] = {key_of(fmaxf(best[0], best[1])), key_of(fmaxf(best[2], best[3]))};
    from = threshold_of<2, kWarps>(k, a.W, a.W + a.W / 8, sh.scratch);
  } else {
    uint32_t k[kVec];
#pragma unroll
    for (int v = 0; v < kVec; ++v) k[v] = key_of(best[v]);
    from = threshold_of<kVec, kWarps>(k, a.W, a.W + a.W / 8, sh.scratch);
  }
  if (!from) from = kNone + 1;
  float M = sh.m[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) M = fmaxf(M, sh.m[w]);
  const float ws = warp_sum(m > -INFINITY ? s * rescale(m, M) : 0.f);
  if (lane == 0) sh.s[warp] = ws;
  const float least = value_of(from);
  // The candidates among kVec vectors, logits at(q, j) of the tokens from t(q) on (those of the bits ok(q)), into the list: places for all
  // of a thread's at once.
  const auto keep = [&](auto&& at, int q, int j, auto&& t, int place) {
    if (place >= kList) return;
    sh.key[place] = key_of(fminf(at(q, j), In<TYPE>::value(In<TYPE>::MOST)));
    sh.tok[place] = t(q) + j;
  };
  const auto gather = [&](auto&& at, auto&& ok, auto&& t) {
    uint32_t hits[kVec];
    int all = 0;
#pragma unroll
    for (int q = 0; q < kVec; ++q) {
      hits[q] = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) hits[q] |= (at(q, j) >= least ? 1u : 0u) << j;
      hits[q] &= ok(q);
      all += __popc(hits[q]);
    }
    if (!all) return;
    int place = atomicAdd(&sh.n, all);
#pragma unroll
    for (int q = 0; q < kVec; ++q) {
      if (!hits[q]) continue;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (hits[q] >> j & 1) keep(at, q, j, t, place++);
    }
  };
  const int tiles = (end - begin + TILE - 1) / TILE;
  if (nothing) {   // (nothing is allowed in the row)
  } else if (tiles == 1) {   // (the tile is at hand, where the warp has any of it)
    if (m > -INFINITY)
      gather([&](int q, int j) { return x.at(q, j); }, [&](int q) { return best[q] >= least ? 0xffffffffu : 0u; }, [&](int q) { return token(begin, q); });
  } else {
    int one = 0, every = 0;   // places to be read in the tile with the maximum, in every tile
#pragma unroll
    for (int v = 0; v < kVec; ++v) {
      every += second[v] >= least;
      one += best[v] >= least && !(second[v] >= least);
    }
    if (one | every) {
      const int at = atomicAdd(&sh.n_reads, one | every << 16);
      int front = at & 0xffff, back = kGroups - (at >> 16);
#pragma unroll
      for (int v = 0; v < kVec; ++v)
        if (best[v] >= least) {
          if (second[v] >= least) sh.read[--back] = token(0, v);
          else sh.read[front++] = token(where[v], v);
        }
    }
  }
  __syncthreads();
  const int n_one = sh.n_reads & 0xffff, n_every = sh.n_reads >> 16, reads = n_one + n_every * tiles;
  for (int i0 = tid; i0 < reads && *(volatile int*)&sh.n <= kList; i0 += kVec * kThreads) {   // (beyond kList it stays so)
    uint32_t w[kVec][4], ok[kVec];
    int t[kVec];
#pragma unroll
    for (int q = 0; q < kVec; ++q) {
      const int i = i0 + q * kThreads;
      t[q] = end;
      if (i < n_one) {
        t[q] = sh.read[i];
      } else if (i < reads) {
        const int tile = (i - n_one) / n_every;
        t[q] = begin + tile * TILE + sh.read[kGroups - 1 - (i - n_one - tile * n_every)];
      }
      vector(t[q], w[q]);
      ok[q] = allowed && t[q] < end ? __ldg(allowed + (t[q] >> 5)) >> (t[q] & 31) : 0xffffffffu;
    }
    gather([&](int q, int j) { return vector_at<TYPE>(w[q], j); }, [&](int q) { return ok[q]; }, [&](int q) { return t[q]; });
  }
  __syncthreads();
  const long long at = (long long)row * a.pieces + piece;
  int n = sh.n;
  const auto hand_on = [&](int i, int to) { a.cand[at * a.cap + to] = make_uint2(__float_as_uint(value_of(sh.key[i])), (uint32_t)sh.tok[i]); };
  const auto hand_on_best = [&] {   // what is at or above a bound among those of the list; false: too many are equal
    uint32_t k[kList / kThreads];
#pragma unroll
    for (int q = 0; q < kList / kThreads; ++q) k[q] = q * kThreads + tid < n ? sh.key[q * kThreads + tid] : 0u;
    const uint32_t bound = threshold_of<kList / kThreads, kWarps>(k, a.W, a.cap, sh.scratch);
    int left = 0, mine = 0;
#pragma unroll
    for (int q = 0; q < kList / kThreads; ++q) {
      left += __syncthreads_count(k[q] >= bound);
      mine += k[q] >= bound;
    }
    if (left > a.cap) return false;
    if (tid == 0) sh.n = 0;
    __syncthreads();
    int to = mine ? atomicAdd(&sh.n, mine) : 0;
#pragma unroll
    for (int q = 0; q < kList / kThreads; ++q)
      if (k[q] >= bound) hand_on(q * kThreads + tid, to++);
    n = left;
    return true;
  };
  if (n <= a.cap || n > kList || !hand_on_best()) {
    if (n > a.cap) {
      __syncthreads();
      put_exactly<TYPE>(in, allowed, begin, end, from, key_of(M), a.W, sh);
      n = sh.n;
    }
    for (int i = tid; i < n; i += kThreads) hand_on(i, i);
  }
  for (int i = n + tid; i < a.cap; i += kThreads) a.cand[at * a.cap + i] = make_uint2(0xff800000u, 0u);   // (-infinity: none)
  if (tid == 0) {
    float all = 0.f;
    for (int w = 0; w < kWarps; ++w) all += sh.s[w];   // (in one order)
    a.head[at] = {M, all};
  }
}

// A candidate of a request: equal scores, the lower row first, then the larger logit, then the lower token.
struct Entry {
  unsigned long long score;   // (as an ordered key)
  unsigned long long rest;    // ~row, logit's key
  uint32_t tok;
};
__device__ __forceinline__ bool before(const Entry& a, const Entry& b) {
  return a.score > b.score || (a.score == b.score && (a.rest > b.rest || (a.rest == b.rest && a.tok < b.tok)));
}

// n log 2 + log(s 2^-32) + more to 2^-29, s > 0.  With s = 2^e f, f in [2/3, 4/3): log f = 2 atanh z = 2 (z + z^3 / 3 + ..),
// z = (f - 1) / (f + 1), |z| <= 1/5; z in two parts (its quotient and what that leaves, times the derivative 1 / (1 - z^2)), the rest of the
// series in one.
__device__ __forceinline__ Two log_of(unsigned long long s, int n, float more) {
  int e = 63 - __clzll(s);
  const unsigned long long f = s << (63 - e);                       // 1.f in 64 bits
  float hi = (float)(uint32_t)(f >> 40) * 0x1p-23f, lo = (float)(uint32_t)(f >> 16 & 0xffffff) * 0x1p-47f;   // (24 bits each)
  if (hi >= 4.f / 3.f) hi *= 0.5f, lo *= 0.5f, ++e;
  const float up = hi - 1.f, down = hi + 1.f, down_lo = (hi - (down - 1.f)) + lo;
  const float z = __fdividef(up, down);
  const float z_lo = __fdividef(fmaf(-z, down, up) + (lo - z * down_lo), down), q = z * z;
  float p = 1.f / 13.f;
  p = fmaf(p, q, 1.f / 11.f);
  p = fmaf(p, q, 1.f / 9.f);
  p = fmaf(p, q, 1.f / 7.f);
  p = fmaf(p, q, 1.f / 5.f);
  p = fmaf(p, q, 1.f / 3.f);
  const float k = (float)(n + e - 32), twos = k * kLn2Hi;
  const float low = fmaf(k, kLn2Hi, -twos) + k * kLn2Lo + fmaf(z + z, q * p, (z_lo + z_lo) * (1.f + q)) + more;
  return add_low(two_sum(twos, z + z), low);
}

// score = cum + ((x - off) - more)
struct alignas(16) Row {
  Two off, more;
  float cum;
  int final;   // the one token of an ended beam; -1
  int pad[2];
  __device__ __forceinline__ Two score(float x) const {
    if (final >= 0) return {cum, 0.f};
    Two t = two_sum(x, -off.hi);
    t.lo -= off.lo;
    if (more.hi != 0.f) {
      const float lo = t.lo - more.lo;
      t = two_sum(t.hi, -more.hi);
      t.lo += lo;
    }
    return add_low(two_sum(cum, t.hi), t.lo);
  }
};

// The same in 32 bits for a first look: bias + x, off by 2^-21 (|that| + size) at most; size < 0: the beam has ended.
struct Quick {
  float bias, size;
};

constexpr int kMostCtas = 304, kManyPieces = kMostCtas / 3 + 1;   // of the first launch where rows are in pieces; rows of three pieces or more
// Few candidates (places of a request's lists) are ranked by a CTA of 256, whose barriers and instructions are fewer: ten rows of 33024, W = 10,
// 11.3 -> 10.8 us, 320 rows 16.5 -> 15.5; 10240 places of 80 beams need the 1024 threads.  The requests' average decides: one of 3001 beams
// among 99 of one takes twice as long as alone (V = 300, W = 10: 224 and 93 us).
constexpr int kFewPlaces = 4096;
constexpr int kRows = 256;   // that shared memory holds (of more: device memory)
template <int T>
struct RankShared {   // of T threads
  unsigned long long score[2 * T], rest[2 * T];
  uint32_t tok[2 * T];
  uint32_t scratch[3 * T / 32];
  float top[kManyPieces];   // rows' maxima, on the way to their logarithms
  Row row[kRows];
  Quick quick[kRows];
  Entry best[kMaxWidth];
  int n, hits[2];
};

// Ranks the list's n entries and hands each that is among the W best to put(rank, entry).  Every thread of the CTA; several threads
// an entry, neighbours in a warp.
template <int T, class Put>
__device__ __forceinline__ void rank_list(const RankShared<T>& sh, int n, int W, Put&& put) {
  int share = 32;   // threads an entry
  while (share > 1 && share * n > T) share >>= 1;
  const int per = T / share, sub = threadIdx.x & (share - 1), mine = threadIdx.x / share;
  for (int j0 = 0; j0 < n; j0 += per) {
    if (j0 + (threadIdx.x & ~31) / share >= n) break;   // (the warp has none)
    const int j = j0 + mine;
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

template <int T>
__global__ void __launch_bounds__(T, 1) beam_rank_kernel(const __grid_constant__ SelectArgs a) {
  extern __shared__ __align__(16) unsigned char raw[];
  RankShared<T>& sh = *reinterpret_cast<RankShared<T>*>(raw);
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r0 = max(max(0, __ldg(a.cu)), __ldg(a.cu + b));
  const int r1 = min(min(a.R, __ldg(a.cu + a.n_req)), __ldg(a.cu + b + 1));
  const int lists = max(0, r1 - r0) * a.pieces;
  if (tid == 0) sh.n = sh.hits[0] = 0;
  // (the first T rows' inputs, before the sums are there)
  const float my_cum = a.score && r0 + tid < r1 ? __ldg(a.score + r0 + tid) : 0.f;
  const int my_final = a.final && r0 + tid < r1 ? __ldg(a.final + r0 + tid) : -1;
  pdl_wait();
  // Candidates: a thread has place `at` of list my_list and of every at_once-th list from there; kHold of them in a round, the
  // first of which are under way while the rows' sums are made.
  const int at_once = T / a.cap, at = tid & (a.cap - 1), my_list = tid / a.cap;
  constexpr int kHold = 16, kBatch = 8;
  const auto fetch = [&](int l) { return l < lists ? a.cand[((long long)r0 * a.pieces + l) * a.cap + at] : make_uint2(0xff800000u, 0u); };
  uint2 c[kBatch];
#pragma unroll
  for (int q = 0; q < kBatch; ++q) c[q] = fetch(q * at_once + my_list);
  const auto row_of = [&](int l) { return r0 + (a.pieces == 1 ? l : (int)__umulhi((unsigned)l, a.per_piece)); };
  const auto row_at = [&](int r) -> Row& { return r - r0 < kRows ? sh.row[r - r0] : a.rows[r]; };
  const auto quick_at = [&](int r) -> Quick& { return r - r0 < kRows ? sh.quick[r - r0] : a.quick[r]; };
  // A row's maximum and sum from its pieces, many by a warp, few by a thread; then its logarithm.
  // (Sums as multiples of 2^-32, whole numbers: a row's is at least 0.7 and at most 1.5 times its length.)
  const auto whole = [&](float s) { return (unsigned long long)(s * 0x1p32f); };
  const auto set_row = [&](int r, float M, unsigned long long s) {   // r: r0 + tid and every T-th from there
    const bool first = r - r0 < T, near = fabsf(M) < kFar;
    Row w = {};
    w.cum = first ? my_cum : a.score ? __ldg(a.score + r) : 0.f;
    w.final = first ? my_final : a.final ? __ldg(a.final + r) : -1;
    if (s) {   // (no sum: no candidates; an ended beam's means nothing)
      const Two l = log_of(s, near ? (int)unit_of(M) : 0, near ? -M * kEta : 0.f);
      if (near) w.off = l;
      else w.off = {M, 0.f}, w.more = l;
    }
    row_at(r) = w;
    Quick q = {w.cum - w.off.hi - w.more.hi, fabsf(w.cum) + fabsf(w.off.hi) + fabsf(w.more.hi)};
    // (score and maximum near the largest number: their difference may pass it, a candidate's score need not)
    if (fabsf(w.cum) < INFINITY && !(fabsf(q.bias) < INFINITY)) q = {0.f, INFINITY};
    quick_at(r) = w.final >= 0 ? Quick{w.cum, -1.f} : q;
  };
  if (a.pieces <= 2) {
    for (int r = r0 + tid; r < r1; r += T) {
      const Header* h = a.head + (long long)r * a.pieces;
      const float m0 = h[0].m, s0 = h[0].s, m1 = a.pieces > 1 ? h[1].m : -INFINITY, s1 = a.pieces > 1 ? h[1].s : 0.f;
      const float M = fmaxf(m0, m1);
      set_row(r, M, M > -INFINITY ? whole(s0 * rescale(m0, M)) + whole(s1 * rescale(m1, M)) : 0ull);
    }
  } else {
    // (there are fewer than kManyPieces rows of three pieces or more; their sums wait in the list's place)
    for (int r = r0 + warp; r < r1; r += T / 32) {
      const Header* h = a.head + (long long)r * a.pieces;
      const float m0 = lane < a.pieces ? h[lane].m : -INFINITY, s0 = lane < a.pieces ? h[lane].s : 0.f;
      float M = m0;
      for (int p = lane + 32; p < a.pieces; p += 32) M = fmaxf(M, h[p].m);
      M = warp_max(M);
      unsigned long long s = m0 > -INFINITY ? whole(s0 * rescale(m0, M)) : 0ull;
      for (int p = lane + 32; p < a.pieces; p += 32)
        if (h[p].m > -INFINITY) s += whole(h[p].s * rescale(h[p].m, M));
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (lane == 0) {
        sh.top[r - r0] = M;
        sh.score[r - r0] = s;
      }
    }
    __syncthreads();
    if (tid < r1 - r0) set_row(r0 + tid, sh.top[tid], sh.score[tid]);
  }
  __syncthreads();
  // in `high` and `low` what the score of candidate c of list l is between, if it has one there
  const auto look = [&](int l, const uint2& c, float& high, float& low) {
    const int r = row_of(l);
    const Quick w = quick_at(r);
    float y = w.bias + __uint_as_float(c.x), e = 0x1p-21f * (fabsf(y) + w.size);
    if (w.size < 0.f) {
      if (at != 0 || l != (r - r0) * a.pieces) return;
      y = w.bias, e = 0.f;
    }
    high = y + e, low = fmaxf(low, y - e);   // (a NaN is passed over)
  };
  float hi[kHold];   // of a round's candidates: not above it
  float g = -INFINITY;
  const auto round = [&](int l0) {
#pragma unroll
    for (int q0 = 0; q0 < kHold; q0 += kBatch) {
#pragma unroll
      for (int q = 0; q < kBatch; ++q) hi[q0 + q] = -INFINITY;
      if (l0 + q0 * at_once >= lists) continue;
      if (l0 || q0) {
#pragma unroll
        for (int q = 0; q < kBatch; ++q) c[q] = fetch(l0 + (q0 + q) * at_once + my_list);
      }
#pragma unroll
      for (int q = 0; q < kBatch; ++q)
        if (l0 + (q0 + q) * at_once + my_list < lists) look(l0 + (q0 + q) * at_once + my_list, c[q], hi[q0 + q], g);
    }
  };
  const int per_round = kHold * at_once;
  for (int l0 = 0; l0 < lists; l0 += per_round) round(l0);
  // what is below `from` is not among the W best: the W-th of the threads' best
  const uint32_t group[1] = {key_of(g)}, bound = threshold_of<1, T / 32>(group, a.W, a.W + a.W / 8, sh.scratch);
  float from = bound ? value_of(bound) : -INFINITY;
  Entry worst = {0, 0, 0};   // what comes after it is not among the W best: the W-th of those known, once there are many
  const auto put = [&](int l) {
    uint2 x = fetch(l);
    const int r = row_of(l);
    const Row& w = row_at(r);
    if (w.final >= 0) x = make_uint2(0u, (uint32_t)w.final);
    const Two y = w.score(__uint_as_float(x.x));
    const Entry e = {key_of(y), (unsigned long long)~(uint32_t)r << 32 | key_of(__uint_as_float(x.x)), x.y};
    if (!(y.hi > -INFINITY) || !before(e, worst)) return;
    const int to = atomicAdd(&sh.n, 1);
    sh.score[to] = e.score;
    sh.rest[to] = e.rest;
    sh.tok[to] = e.tok;
  };
  for (int l0 = 0, turn = 0; l0 < lists; l0 += per_round, turn ^= 1) {
    if (lists > per_round) {
#pragma unroll
      for (int q = 0; q < kBatch; ++q) c[q] = fetch(q * at_once + my_list);   // (round 0 takes these)
      round(l0);
    }
    uint32_t hits = 0;
#pragma unroll
    for (int q = 0; q < kHold; ++q) hits |= (hi[q] >= from && hi[q] > -INFINITY ? 1u : 0u) << q;
    const int mine = __reduce_add_sync(0xffffffffu, __popc(hits));
    if (lane == 0 && mine) atomicAdd(&sh.hits[turn], mine);
    __syncthreads();
    const int all = sh.hits[turn], had = sh.n;
    if (tid == 0) sh.hits[turn ^ 1] = 0;
    if (had + all <= 2 * T) {
      __syncthreads();   // (everyone knows `had`)
#pragma unroll 1
      for (; hits; hits &= hits - 1) put(l0 + (__ffs(hits) - 1) * at_once + my_list);
    } else {
      // Too many, most of them equal: a quarter of the threads at a time, of which the W best stay, and what comes after those is left
      // out (later rows come after equal ones): an order of fewer, of a quarter of the work.  What the rounds before left may fill the list
      // to its end, so it is ranked before the first share (q = -1): fewer than W + T / 4 are there whenever one is put in.
      static_assert(kMaxWidth + T / 2 <= 2 * T, "a share more than the list was ranked at");
#pragma unroll 1
      for (int q = -1; q < 4 * kHold; ++q) {
        __syncthreads();
        if (q >= 0 && hits >> q / 4 & 1 && tid / (T / 4) == q % 4) put(l0 + q / 4 * at_once + my_list);
        __syncthreads();
        const int n = sh.n;
        if (n < a.W + T / 4) continue;
        rank_list(sh, n, a.W, [&](int r, const Entry& e) { sh.best[r] = e; });
        __syncthreads();
        for (int j = tid; j < a.W; j += T) sh.score[j] = sh.best[j].score, sh.rest[j] = sh.best[j].rest, sh.tok[j] = sh.best[j].tok;
        if (tid == 0) sh.n = a.W;
        worst = sh.best[a.W - 1];
        from = fmaxf(from, value_of((uint32_t)(worst.score >> 32)));
      }
    }
    __syncthreads();
  }
  __syncthreads();
  const int n = sh.n;
  const long long o = (long long)b * a.W;
  rank_list(sh, n, a.W, [&](int r, const Entry& e) {
    a.token[o + r] = (int)e.tok;
    a.parent[o + r] = (int)~(uint32_t)(e.rest >> 32);
    a.out_score[o + r] = value_of((uint32_t)(e.score >> 32));
  });
  for (int j = n + tid; j < a.W; j += T) {
    a.token[o + j] = -1;
    a.parent[o + j] = -1;
    a.out_score[o + j] = -INFINITY;
  }
}

constexpr int kTile = In<ATSPEED_F32>::TILE;
// Pieces of a row: up to two CTAs an SM, none shorter than four tiles (of 32-bit logits, whatever the type).  Each costs a bound and more
// candidates to rank.  us for 1 / 2 / 4 / 9 / 17 pieces of 33024 logits: 10 rows 12.4 / 11.1 / 10.6 / 10.3 / 11.2, 16 rows 13.2 / 11.5 /
// 11.4 / 12.1 / 12.5, 320 rows 15.9 / 16.0 / 20.2 / 25.6 / 43, 3840 rows 100 / 112 / 155 / 357 / 580.
static_assert(kManyPieces <= 256, "a thread a row of several pieces");
int pieces_of(int R, int V) {
  const long long tiles = (V + kTile - 1LL) / kTile, most = std::max(1LL, std::min((tiles + 3) / 4, (long long)kMostCtas / R));
  const long long span = (tiles + most - 1) / most;
  return (int)((tiles + span - 1) / span);
}
int cap_of(int W) {   // candidates that a piece hands on at most: a power of two
  int cap = 32;
  while (cap < W + W / 2 + 8) cap *= 2;
  return cap;
}

struct Layout {
  int pieces;
  size_t cand, rows, quick, bytes;
};
Layout layout_of(int R, int V, int W) {
  Layout l;
  l.pieces = pieces_of(R, V);
  const size_t n = (size_t)R * l.pieces;
  l.cand = n * sizeof(Header);
  l.rows = (l.cand + n * cap_of(W) * sizeof(uint2) + 15) / 16 * 16;
  l.quick = l.rows + (size_t)R * sizeof(Row);
  l.bytes = l.quick + (size_t)R * sizeof(Quick);
  return l;
}

}  // namespace
}  // namespace atspeed

using namespace atspeed;

extern "C" size_t atspeed_op_beam_select_workspace(int R, int vocab, int width) {
  return R > 0 && vocab > 0 && width > 0 ? layout_of(R, vocab, std::min(width, kMaxWidth)).bytes : 0;
}

extern "C" atspeed_status atspeed_op_beam_select(atspeed_stream stream, const atspeed_beams* beams, void* d_ws) {
  if (!beams) return ATSPEED_E_ARG;
  const atspeed_beams& s = *beams;
  const int R = s.R, vocab = s.vocab, width = s.width;
  if (!s.d_logits || !s.d_cu_beam || !s.d_token || !s.d_parent || !s.d_out_score || !d_ws || R <= 0 || vocab <= 0 || s.n_req <= 0 ||
      width <= 0 || s.ld < vocab || !dtype_size(s.type) || reinterpret_cast<uintptr_t>(s.d_logits) % dtype_size(s.type) ||
      !aligned16(d_ws) || (s.norm != ATSPEED_NORM_MASKED && s.norm != ATSPEED_NORM_FULL) ||
      (s.d_state && (!s.d_grammar || s.n_states <= 0 || s.grammar_stride < (vocab + 31LL) / 32)))
    return ATSPEED_E_ARG;
  const Layout l = layout_of(R, vocab, std::min(width, kMaxWidth));
  if (width > kMaxWidth || vocab > 1 << 30 || (long long)R * l.pieces > 0x7fffffffLL) return ATSPEED_E_SHAPE;
  const long long rows = 4ll * R, places = 4ll * s.n_req * width;   // bytes
  const Span in[] = {{s.d_logits, ((R - 1) * s.ld + vocab) * dtype_size(s.type)}, {s.d_cu_beam, 4ll * s.n_req + 4}, {s.d_score, rows},
                     {s.d_final, rows}, {s.d_state, rows},
                     {s.d_state ? s.d_grammar : nullptr, 4 * ((s.n_states - 1ll) * s.grammar_stride + (vocab + 31ll) / 32)}};
  const Span out[] = {{s.d_token, places}, {s.d_parent, places}, {s.d_out_score, places}};
  if (outputs_overlap(out, in)) return ATSPEED_E_ARG;   // (a request's places are written while another's rows are read)
  SelectArgs a = {};
  a.logits = s.d_logits, a.ld = s.ld, a.R = R, a.V = vocab, a.n_req = s.n_req, a.W = width, a.pieces = l.pieces, a.cap = cap_of(width);
  a.span = (int)(((vocab + (long long)l.pieces - 1) / l.pieces + kTile - 1) / kTile * kTile);
  a.score = s.d_score, a.final = s.d_final, a.cu = s.d_cu_beam, a.state = s.d_state, a.grammar = s.d_grammar;
  a.grammar_stride = s.grammar_stride, a.n_states = s.d_state ? s.n_states : 0, a.full = s.norm == ATSPEED_NORM_FULL;
  a.per_piece = l.pieces > 1 ? (uint32_t)((0x100000000ll + l.pieces - 1) / l.pieces) : 0u;
  a.token = s.d_token, a.parent = s.d_parent, a.out_score = s.d_out_score;
  char* ws = static_cast<char*>(d_ws);
  a.head = reinterpret_cast<Header*>(ws), a.cand = reinterpret_cast<uint2*>(ws + l.cand);
  a.rows = reinterpret_cast<Row*>(ws + l.rows), a.quick = reinterpret_cast<Quick*>(ws + l.quick);
  const int grid = R * l.pieces;
  const bool aligned = aligned16(s.d_logits) && s.ld * dtype_size(s.type) % 16 == 0;
  static std::atomic<unsigned long long> ready[6];
  const auto go = [&](auto kernel, int i) {
    if (smem_attr_once(ready[i], kernel, (int)sizeof(PieceShared)) != cudaSuccess) return ATSPEED_E_CUDA;
    kernel<<<grid, kThreads, sizeof(PieceShared), (cudaStream_t)stream>>>(a);
    return launch_status();
  };
  const atspeed_status launched =
      s.type == ATSPEED_F32    ? aligned ? go(beam_pieces_kernel<ATSPEED_F32, true>, 0) : go(beam_pieces_kernel<ATSPEED_F32, false>, 1)
      : s.type == ATSPEED_BF16 ? aligned ? go(beam_pieces_kernel<ATSPEED_BF16, true>, 2) : go(beam_pieces_kernel<ATSPEED_BF16, false>, 3)
      : aligned                ? go(beam_pieces_kernel<ATSPEED_F16, true>, 4)
                               : go(beam_pieces_kernel<ATSPEED_F16, false>, 5);
  if (launched != ATSPEED_OK) return launched;
  // The ranking may start while the last of the pieces are read, and waits for them.
  const auto rank = [&](auto kernel, int threads, size_t shared, std::atomic<unsigned long long>& done) {
    if (smem_attr_once(done, kernel, (int)shared) != cudaSuccess) return ATSPEED_E_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(s.n_req), cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = shared, cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr, cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a) == cudaSuccess ? ATSPEED_OK : ATSPEED_E_CUDA;
  };
  static std::atomic<unsigned long long> done[2];
  const long long looked_at = (long long)grid * a.cap / s.n_req;   // candidates' places, a request's on average
  return width <= 64 && looked_at <= kFewPlaces ? rank(beam_rank_kernel<256>, 256, sizeof(RankShared<256>), done[0])
                                             : rank(beam_rank_kernel<1024>, 1024, sizeof(RankShared<1024>), done[1]);
}
