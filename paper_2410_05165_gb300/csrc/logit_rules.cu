// Penalties, biases, grammar masks and temperature on next-token logits (atspeed_op_adjust_logits).
//   c(v) = occurrences of v in the request's output and on the row's path in its tree, seen(v) = c(v) > 0 or v in the prompt
//   x <- seen ? (x > 0 ? x / rep : x * rep) : x;  x <- x - freq c - pres [c > 0] + bias(v);  forbidden: -inf;  x <- x / temp
// Bound: HBM (each logit read and written once).  3840 rows of 33024 (32 bits) take 240 us, 4.2 TB/s; with the temperature alone
// 172, a plain copy 152.  509 rows of 100003 (bf16) with histories of up to 8000 tokens take 117 us, 1.8 TB/s: there each piece
// of a row goes through the whole history, whose loads wait for the request's, and a CTA has too few bytes under way meanwhile
// (without histories 85 us, a copy 40).  Pieces twice as long leave two CTAs an SM for the table's sake and take 154 us.
//
// The penalties and biases touch some hundred tokens of a vocabulary of tens of thousands.  So a warp streams its 512 tokens of
// a row (temperature and the grammar's bits: a few instructions a logit) and then does the touched ones among them again,
// each from its own logit: they stand in a list, made once per request for several of its rows, with the counts in a table
// of one word a token.  A row's path in its tree joins the counts and the list for that row.  The table is the warp's own, so
// that a row takes no barrier of the CTA (one a row: 3840 rows of 33024 took 270 us); counts looked up for every logit cost
// 160 instructions per 128 logits (403 us).
// Rows are read and written at multiples of 16 bytes whatever their start: a warp's tokens of a row begin up to 7 early, and the
// words of 16 tokens at a border are held by both warps.
#include <algorithm>

#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSub = 512;               // tokens of a warp
constexpr int kRegion = kSub + 16;      // .. and its words: from 8 tokens before the first
constexpr int kChunk = kSub * kWarps;   // tokens of a CTA
constexpr int kBatch = 8;               // entries of a history that a thread has under way
constexpr uint32_t kPrompt = 1u << 31, kListed = 1u << 30;   // flags of a token's word; below them its count in the output

struct RulesArgs {
  const void* in;
  void* out;
  long long ld_in, ld_out;
  int R, V, n, rows, words;   // rows: consecutive rows a CTA takes
  unsigned groups, chunks;    // of rows, of the vocabulary
  bool in_place, by_row;      // by_row: neighbouring CTAs take other rows, not other pieces
  const int* req;
  const uint32_t* mask;
  const int* state;
  atspeed_logit_rules r;
};

template <int TYPE>
struct Logit {   // values of one 16-byte access
  static constexpr int N = TYPE == ATSPEED_F32 ? 4 : 8;
  static constexpr int SIZE = 16 / N;
  static __device__ __forceinline__ float at(const uint4& v, int j) {
    const uint32_t w = (&v.x)[TYPE == ATSPEED_F32 ? j : j / 2];
    if constexpr (TYPE == ATSPEED_F32) return __uint_as_float(w);
    else return j & 1 ? unpack2(w, TYPE == ATSPEED_F16).y : unpack2(w, TYPE == ATSPEED_F16).x;
  }
  static __device__ __forceinline__ void store1(char* p, float x) {
    if constexpr (TYPE == ATSPEED_F32) *reinterpret_cast<float*>(p) = x;
    else *reinterpret_cast<uint16_t*>(p) = (uint16_t)pack2(x, 0.f, TYPE == ATSPEED_F16);
  }
};

// The rules of a request that a multiplication expresses: 1 / temperature and 1 / repetition are rounded once per request
// (the quotient is within 1.5 units in the last place of the exact one, in 32 bits); where the reciprocal leaves the
// normal range, or would round there, the division is done.
struct Factors {
  float rep, rep_inv, freq, pres, temp, temp_inv;
  bool divide;
};
__device__ __forceinline__ bool usual(float x) { return x > 0x1p-100f && x < 0x1p100f; }

template <int IN, int OUT>
__global__ void __launch_bounds__(kThreads, 4) adjust_logits_kernel(const __grid_constant__ RulesArgs a) {
  using I = Logit<IN>;
  using O = Logit<OUT>;
  constexpr int N = I::N, U = kSub / (32 * N);
  extern __shared__ __align__(16) uint32_t sm[];
  __shared__ int s_n[kWarps];   // tokens in a warp's list
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool biased = a.r.d_bias_off != nullptr;
  // a warp's words: counts, its list (16 bits an entry), with biases the number + 1 of a token's entry, in place the listed
  // tokens' logits
  const int words = kRegion + kRegion / 2 + (biased ? kRegion : 0) + (a.in_place ? kRegion : 0);
  uint32_t* cnt = sm + warp * words;
  uint16_t* list = reinterpret_cast<uint16_t*>(cnt + kRegion);
  uint32_t* bias = cnt + kRegion + kRegion / 2;
  uint32_t* raw = bias + (biased ? kRegion : 0);
  const int v0 = (int)(a.by_row ? blockIdx.x / a.groups : blockIdx.x % a.chunks) * kChunk, s0 = v0 + warp * kSub;
  const int r0 = (int)(a.by_row ? blockIdx.x % a.groups : blockIdx.x / a.chunks) * a.rows, r1 = min(a.R, r0 + a.rows);
  const auto in_row = [&](int row) { return static_cast<const char*>(a.in) + (long long)row * a.ld_in * I::SIZE; };
  // the warp's first token in a row: the last one not past s0 whose address is a multiple of 16
  const auto begin = [&](const char* in) { return s0 - (int)((reinterpret_cast<uintptr_t>(in) / I::SIZE + s0) & (N - 1)); };
  const auto one = [&](const char* in, int t) {   // a logit's bits
    if constexpr (I::SIZE == 4) return reinterpret_cast<const uint32_t*>(in)[t];
    else return (uint32_t)reinterpret_cast<const uint16_t*>(in)[t];
  };
  const auto value = [](uint32_t bits) {
    if constexpr (IN == ATSPEED_F32) return __uint_as_float(bits);
    else return unpack2(bits, IN == ATSPEED_F16).x;
  };
  uint4 x[U];
  const auto load = [&](int row) {
    const char* in = in_row(row);
    const int w0 = begin(in), t0 = w0 + lane * N;
    if (w0 >= 0 && w0 + kSub <= a.V) {
      const uint4* v = reinterpret_cast<const uint4*>(in + (long long)t0 * I::SIZE);
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = __ldcs(v + 32 * u);
    }
  };
  const auto request_of = [&](int row) {
    const int b = row < r1 ? __ldg(a.req + row) : -1;
    return b < a.n ? b : -1;
  };
  const auto state_of = [&](int row) { return a.state && a.r.d_grammar && row < r1 ? __ldg(a.state + row) : -1; };
  load(r0);
  for (int i = lane; i < kRegion / 4; i += 32) reinterpret_cast<uint4*>(cnt)[i] = make_uint4(0, 0, 0, 0);
  if (biased)
    for (int i = lane; i < kRegion / 4; i += 32) reinterpret_cast<uint4*>(bias)[i] = make_uint4(0, 0, 0, 0);
  if (lane == 0) s_n[warp] = 0;
  // the request whose counts the table holds, the tokens it lists, its first bias entry, its tree's first token and length
  int held = -2, base = 0, k0 = 0, q0 = 0, q_len = 0;
  Factors f = {1.f, 1.f, 0.f, 0.f, 1.f, 1.f, false};
  // (a row's request and state are read a row ahead: what they lead to takes long enough)
  const auto bits_of = [&](int row) {   // a lane's word of a row's mask
    return a.mask && row < r1 && lane < a.words ? __ldg(a.mask + (long long)row * a.words + lane) : 0u;
  };
  int b = request_of(r0), st = state_of(r0);
  uint32_t mask_bits = bits_of(r0);
  for (int row = r0; row < r1; ++row) {
    const int b_next = request_of(row + 1), st_next = state_of(row + 1);
    const uint32_t bits_next = bits_of(row + 1);
    if (b != held) {
      held = b;
      f = {1.f, 1.f, 0.f, 0.f, 1.f, 1.f, false};
      int h0 = 0, h1 = 0, p = 0, k1 = 0;
      k0 = 0, q_len = 0;
      if (b >= 0) {
        if (a.mask && a.r.d_tree_tok) q0 = __ldg(a.r.d_cu_q + b), q_len = __ldg(a.r.d_cu_q + b + 1) - q0;
        if (a.r.d_hist) {
          h0 = __ldg(a.r.d_hist_off + b), h1 = __ldg(a.r.d_hist_off + b + 1);
          p = h0 + (a.r.d_prompt_len ? __ldg(a.r.d_prompt_len + b) : 0);
        }
        if (biased) k0 = __ldg(a.r.d_bias_off + b), k1 = __ldg(a.r.d_bias_off + b + 1);
        if (a.r.d_repetition) f.rep = __ldg(a.r.d_repetition + b);
        if (a.r.d_frequency) f.freq = __ldg(a.r.d_frequency + b);
        if (a.r.d_presence) f.pres = __ldg(a.r.d_presence + b);
        if (a.r.d_temperature) f.temp = __ldg(a.r.d_temperature + b);
        if (!(f.temp > 0.f)) f.temp = 1.f;
        f.rep_inv = 1.f / f.rep;
        f.temp_inv = 1.f / f.temp;
        f.divide = !usual(f.rep) || !usual(f.temp);
      }
      for (int e = lane; e < base; e += 32) {   // the words of the request before
        const int i = list[e];
        cnt[i] = 0;
        if (biased) bias[i] = 0;
      }
      if (lane == 0) s_n[warp] = 0;
      __syncthreads();
      // a token's words, with the warp's number, and the second ones if it lies at a border
      const auto each = [&](int v, auto&& go) {
        const int rel = v - v0 + 8;
        if ((unsigned)v >= (unsigned)a.V || (unsigned)rel >= (unsigned)(kChunk + 16)) return;
        const int w = rel / kSub, i = rel % kSub;
        if (w < kWarps) go(w, i);
        if (w > 0 && i < 16) go(w - 1, kSub + i);
      };
      const auto enlist = [&](int w, int i) {
        uint32_t* c = sm + w * words;
        if (!(atomicOr(c + i, kListed) & kListed)) reinterpret_cast<uint16_t*>(c + kRegion)[atomicAdd(&s_n[w], 1)] = (uint16_t)i;
      };
      // (kBatch entries a thread at once; few are among the CTA's tokens, and those are read again.  What is left is counted, not
      // the places: a step past the end of lists that end near 2^31 would come round to negative ones)
      const int* at = a.r.d_hist + h0 + (long long)tid;
      for (int left = h1 - h0 - tid; left > 0; left -= kBatch * kThreads, at += kBatch * kThreads) {
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int v = j * kThreads < left ? __ldg(at + j * kThreads) : -1;
          if ((unsigned)v < (unsigned)a.V && (unsigned)(v - v0 + 8) < (unsigned)(kChunk + 16)) hits |= 1u << j;
        }
#pragma unroll 1
        for (; hits; hits &= hits - 1) {
          const int j = (__ffs(hits) - 1) * kThreads;
          each(__ldg(at + j), [&](int w, int i) {
            if (h1 - left + j < p) atomicOr(sm + w * words + i, kPrompt);
            else atomicAdd(sm + w * words + i, 1u);
            enlist(w, i);
          });
        }
      }
      for (unsigned k = k0 + tid; k < (unsigned)k1; k += kThreads)
        each(__ldg(a.r.d_bias_tok + k), [&](int w, int i) {   // (the later entry)
          atomicMax(sm + w * words + kRegion + kRegion / 2 + i, k - k0 + 1u);
          enlist(w, i);
        });
      __syncthreads();
      base = s_n[warp];
      __syncwarp();   // (every lane has it before a row's path adds to the list)
    }
    const char* in = in_row(row);
    char* out = static_cast<char*>(a.out) + (long long)row * a.ld_out * O::SIZE;
    const int t0 = begin(in);
    const uint32_t* allowed = st >= 0 && st < a.r.n_states ? a.r.d_grammar + st * a.r.grammar_stride : nullptr;
    const auto forbidden = [&](int t) { return allowed && !(__ldg(allowed + (t >> 5)) >> (t & 31) & 1); };
    // the row's path: its tokens among the warp's, counted and listed for this row
    int listed = base;
    const auto walk = [&](auto&& go) {
      for (int w = lane; w < a.words && 32 * w < q_len; w += 32) {
        uint32_t bits = w < 32 ? mask_bits : __ldg(a.mask + (long long)row * a.words + w);
        while (bits) {
          const int j = 32 * w + __ffs(bits) - 1;
          bits &= bits - 1;
          if (j >= q_len) break;
          const int v = __ldg(a.r.d_tree_tok + q0 + j);
          if (v >= max(t0, 0) && v < min(t0 + kSub, a.V)) go(v - s0 + 8);
        }
      }
    };
    bool path = q_len > 0;
    if (path) {
      bool hit = false;
      walk([&](int i) {
        hit = true;
        atomicAdd(cnt + i, 1u);
        if (!(atomicOr(cnt + i, kListed) & kListed)) list[atomicAdd(&s_n[warp], 1)] = (uint16_t)i;
      });
      path = __any_sync(0xffffffffu, hit);
      __syncwarp();
      if (path) listed = *reinterpret_cast<volatile int*>(&s_n[warp]);
    }
    // the listed tokens' logits, before they are overwritten; a lane's first one stays in a register
    const auto token = [&](int e) {   // a listed token, -1: not the warp's in this row
      const int t = s0 - 8 + list[e];
      return t >= t0 && t < t0 + kSub ? t : -1;
    };
    const int my_t = lane < listed ? token(lane) : -1;
    uint32_t my_raw = 0, my_w = 0;
    float my_bias = 0.f;
    bool my_forbidden = false;
    if (my_t >= 0) {
      my_raw = one(in, my_t);
      my_forbidden = forbidden(my_t);
      my_w = cnt[list[lane]];
      if (const uint32_t k = biased ? bias[list[lane]] : 0u) my_bias = __ldg(a.r.d_bias_val + k0 + k - 1);
    }
    if (a.in_place) {
      for (int e = 32 + lane; e < listed; e += 32) {
        const int t = token(e);
        if (t >= 0) raw[e] = one(in, t);
      }
      __syncwarp();
    }
    // every logit by temperature and grammar
    char* to = out + (long long)(t0 + lane * N) * O::SIZE;
    const bool wide = ((reinterpret_cast<uintptr_t>(out) + (long long)t0 * O::SIZE) & 15) == 0;
    if (t0 >= 0 && t0 + kSub <= a.V && wide && !f.divide) {
      // (the bits of a vector begin at the same place of a word in all of the lane's vectors)
      const int t = t0 + lane * N, sh = t & 31;
      const uint32_t* g_at = allowed + (t >> 5);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float y[N];
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = I::at(x[u], j) * f.temp_inv;
        if (allowed) {
          uint32_t g = __ldg(g_at + u * N) >> sh;
          if (sh + N > 32) g |= __ldg(g_at + u * N + 1) << (32 - sh);
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (!(g >> j & 1)) y[j] = -INFINITY;
        }
        if constexpr (OUT == ATSPEED_F32) {
#pragma unroll
          for (int j = 0; j < N; j += 4)
            *reinterpret_cast<float4*>(to + (u * 32 * N + j) * 4) = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
        } else {
          constexpr bool H = OUT == ATSPEED_F16;
          *reinterpret_cast<uint4*>(to + u * 32 * N * 2) =
              make_uint4(pack2(y[0], y[1], H), pack2(y[2], y[3], H), pack2(y[4], y[5], H), pack2(y[6], y[7], H));
        }
      }
    } else {   // a row's ends, an output out of line with its input, an unusual temperature
      for (int t = max(t0, 0) + lane; t < min(t0 + kSub, a.V); t += 32) {
        const float y = value(one(in, t));
        O::store1(out + (long long)t * O::SIZE, forbidden(t) ? -INFINITY : f.divide ? y / f.temp : y * f.temp_inv);
      }
    }
    if (row + 1 < r1) load(row + 1);
    __syncwarp();
    // the listed ones with all rules
    const auto finish = [&](int t, uint32_t logit, uint32_t w, float add, bool forbid) {
      const uint32_t c = w & (kListed - 1);
      float y = value(logit);
      if (c || w & kPrompt) y = y > 0.f ? (f.divide ? y / f.rep : y * f.rep_inv) : y * f.rep;
      if (c) y = y - f.freq * (float)c - f.pres;
      y += add;
      y = f.divide ? y / f.temp : y * f.temp_inv;
      O::store1(out + (long long)t * O::SIZE, forbid ? -INFINITY : y);
    };
    if (my_t >= 0) finish(my_t, my_raw, my_w, my_bias, my_forbidden);
    for (int e = 32 + lane; e < listed; e += 32) {
      const int t = token(e);
      if (t < 0) continue;
      const int i = list[e];
      const uint32_t k = biased ? bias[i] : 0u;
      finish(t, a.in_place ? raw[e] : one(in, t), cnt[i], k ? __ldg(a.r.d_bias_val + k0 + k - 1) : 0.f, forbidden(t));
    }
    __syncwarp();
    // A state past the table allows nothing.  (Here, over what was written: asked for with each logit, it cost 3840 rows of 33024
    // 254 us for 240; like this 243.)
    if (__builtin_expect(st >= a.r.n_states, 0))
      for (int t = max(t0, 0) + lane; t < min(t0 + kSub, a.V); t += 32) O::store1(out + (long long)t * O::SIZE, -INFINITY);
    if (path) {   // the path's tokens leave again
      walk([&](int i) { atomicAdd(cnt + i, ~0u); });
      for (int e = base + lane; e < listed; e += 32) atomicAnd(cnt + list[e], ~kListed);
      if (lane == 0) s_n[warp] = base;
      __syncwarp();
    }
    b = b_next, st = st_next, mask_bits = bits_next;
  }
}

}  // namespace
}  // namespace atspeed

using namespace atspeed;

extern "C" atspeed_status atspeed_op_adjust_logits(atspeed_stream stream, const void* d_logits, atspeed_dtype in_type,
                                                   int64_t ld_in, int R, int vocab, const int32_t* d_req,
                                                   const atspeed_logit_rules* rules, const uint32_t* d_mask, int mask_words,
                                                   const int32_t* d_state, void* d_out, atspeed_dtype out_type,
                                                   int64_t ld_out) {
  if (!d_logits || !d_out || !d_req || !rules || R <= 0 || vocab <= 0 || ld_in < vocab || ld_out < vocab || rules->n_req < 0)
    return ATSPEED_E_ARG;
  const atspeed_logit_rules& r = *rules;
  if (!dtype_size(in_type) || !dtype_size(out_type) || (out_type != in_type && out_type != ATSPEED_F32)) return ATSPEED_E_ARG;
  if (reinterpret_cast<uintptr_t>(d_logits) % dtype_size(in_type) || reinterpret_cast<uintptr_t>(d_out) % dtype_size(out_type))
    return ATSPEED_E_ARG;
  if (d_out == d_logits && (in_type != out_type || ld_in != ld_out)) return ATSPEED_E_ARG;
  if ((r.d_hist && !r.d_hist_off) || (r.d_bias_off && (!r.d_bias_tok || !r.d_bias_val)) ||
      (d_mask && (mask_words <= 0 || !r.d_tree_tok || !r.d_cu_q)) ||
      (d_state && (!r.d_grammar || r.n_states <= 0 || r.grammar_stride < (vocab + 31) / 32)))
    return ATSPEED_E_ARG;
  RulesArgs a = {};
  a.in = d_logits, a.out = d_out, a.ld_in = ld_in, a.ld_out = ld_out;
  a.R = R, a.V = vocab, a.n = r.n_req, a.words = mask_words, a.req = d_req, a.mask = d_mask, a.state = d_state;
  a.r = r;
  if (!d_state) a.r.n_states = 0;
  a.in_place = d_out == d_logits;
  // Pieces of 4096 tokens (7 more for rows that begin between 16-byte addresses).  Rows a CTA: a request's list is made once for
  // those that follow each other, and more CTAs than run at once even out their ends.  us for 1 / 2 / 4 / 8 / 16 rows: 3840 rows of
  // 33024, 240 a request, 328 / 266 / 243 / 244 / 261; 509 rows of 100003, one a request, 117 / 140 / 158 / 178 / 230.
  // Neighbouring CTAs take a row's pieces one after the other (3840 rows: 243, row after row 260), except where every row has
  // a history of its own, whose long ones then spread (509 rows: 123 and 117).  (n_req that counts more requests than the rows
  // are of makes it fewer rows a CTA than would do: slower, not wrong.)
  a.chunks = (unsigned)((vocab + 7LL + kChunk - 1) / kChunk);
  a.rows = std::min(4, std::max(1, R / std::max(1, r.n_req)));
  a.groups = (unsigned)((R + a.rows - 1LL) / a.rows);
  a.by_row = a.rows == 1;
  if ((long long)a.chunks * a.groups > 0x7fffffffLL) return ATSPEED_E_SHAPE;
  const unsigned grid = a.chunks * a.groups;
  const int smem = kWarps * 2 * (kRegion * 3 + (r.d_bias_off ? kRegion * 2 : 0) + (a.in_place ? kRegion * 2 : 0));
  auto go = [&](auto kernel, std::atomic<unsigned long long>& done) {
    if (smem_attr_once(done, kernel, kWarps * kRegion * 14) != cudaSuccess) return ATSPEED_E_CUDA;
    kernel<<<grid, kThreads, smem, (cudaStream_t)stream>>>(a);
    return launch_status();
  };
  static std::atomic<unsigned long long> done[5];
  if (in_type == ATSPEED_F32) return go(adjust_logits_kernel<ATSPEED_F32, ATSPEED_F32>, done[0]);
  if (in_type == ATSPEED_BF16)
    return out_type == ATSPEED_F32 ? go(adjust_logits_kernel<ATSPEED_BF16, ATSPEED_F32>, done[1])
                                   : go(adjust_logits_kernel<ATSPEED_BF16, ATSPEED_BF16>, done[2]);
  return out_type == ATSPEED_F32 ? go(adjust_logits_kernel<ATSPEED_F16, ATSPEED_F32>, done[3])
                                 : go(adjust_logits_kernel<ATSPEED_F16, ATSPEED_F16>, done[4]);
}
