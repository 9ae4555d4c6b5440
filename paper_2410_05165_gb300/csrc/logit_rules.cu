// Penalties, biases, grammar masks and temperature on next-token logits (atspeed_op_adjust_logits).
//   c(v) = occurrences of v in the request's output and on the row's path in its tree, seen(v) = c(v) > 0 or v in the prompt
//   x <- seen ? (x > 0 ? x / rep : x * rep) : x;  x <- x - freq c - pres [c > 0] + bias(v);  forbidden: -inf;  x <- x / temp
// Bound: HBM (each logit read and written once).
//
// A warp owns 1024 tokens of the vocabulary and one word of shared memory for each (its count and whether the prompt has
// it).  A CTA counts a request's history into its warps' words once and walks several rows of that request; a row's path
// is added by each warp to its own words and taken away after, so that rows cost no barrier, and the history is scanned
// once per CTA, not once per row.  Rows are read and written by 16 bytes at addresses that are multiples of 16, whatever the
// row's start is: a warp's 1024 tokens begin up to 7 tokens early, and the words of 16 tokens at a border are held by both.
#include <algorithm>

#include "common.cuh"
#include "gemm.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kWarps = 8;               // of a CTA, at most
constexpr int kSub = 1024;              // tokens of a warp
constexpr int kRegion = kSub + 16;      // .. and its words
constexpr uint32_t kPrompt = 1u << 31;  // the token occurs in the prompt; below it the count in the output

struct RulesArgs {
  const void* in;
  void* out;
  long long ld_in, ld_out;
  int R, V, n, rows, words, subs;   // rows: consecutive rows a CTA takes; subs: warps of a CTA
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
  static __device__ __forceinline__ uint32_t load1(const char* p) {   // one value's bits
    if constexpr (TYPE == ATSPEED_F32) return *reinterpret_cast<const uint32_t*>(p);
    else return *reinterpret_cast<const uint16_t*>(p);
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
__global__ void __launch_bounds__(32 * kWarps) adjust_logits_kernel(const __grid_constant__ RulesArgs a) {
  using I = Logit<IN>;
  using O = Logit<OUT>;
  constexpr int N = I::N, U = kSub / (32 * N);
  extern __shared__ __align__(16) uint32_t sm[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
  const bool biased = a.r.d_bias_off != nullptr;
  uint32_t* cnt = sm + warp * kRegion;                  // this warp's words
  uint32_t* all_bias = sm + a.subs * kRegion;           // index + 1 of a token's bias entry (with biases)
  uint32_t* bias = all_bias + warp * kRegion;
  const int v0 = blockIdx.x * a.subs * kSub, s0 = v0 + warp * kSub;
  const int r0 = blockIdx.y * a.rows, r1 = min(a.R, r0 + a.rows);
  int held = -2, held_shift = 0;   // the request whose counts the words hold, and the tokens they begin early
  Factors f = {1.f, 1.f, 0.f, 0.f, 1.f, 1.f, false};
  for (int row = r0; row < r1; ++row) {
    const char* in = static_cast<const char*>(a.in) + row * a.ld_in * I::SIZE;
    char* out = static_cast<char*>(a.out) + row * a.ld_out * O::SIZE;
    // the warp's first token in this row: the last one not past s0 whose address is a multiple of 16
    const int shift = (int)((reinterpret_cast<uintptr_t>(in) / I::SIZE + s0) & (N - 1));
    const int t0 = s0 - shift;
    uint4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + (lane + 32 * u) * N;
      raw[u] = make_uint4(0, 0, 0, 0);
      if (t >= 0 && t + N <= a.V) {
        raw[u] = __ldcs(reinterpret_cast<const uint4*>(in + (long long)t * I::SIZE));
      } else if (t + N > 0 && t < a.V) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (t + j >= 0 && t + j < a.V) {
            const uint32_t b = I::load1(in + (long long)(t + j) * I::SIZE);
            (&raw[u].x)[j * I::SIZE / 4] |= I::SIZE == 4 ? b : b << (j % 2 * 16);
          }
      }
    }
    int b = a.req[row];
    if (b < 0 || b >= a.n) b = -1;
    if (b != held) {
      // the words begin with this row's first token, so that its reads of them are aligned
      held = b;
      held_shift = (int)((reinterpret_cast<uintptr_t>(in) / I::SIZE + v0) & (N - 1));
      f = {1.f, 1.f, 0.f, 0.f, 1.f, 1.f, false};
      __syncthreads();
      const uint4 zero = make_uint4(0, 0, 0, 0);
      for (int i = tid; i < a.subs * kRegion / 4 * (biased ? 2 : 1); i += threads) reinterpret_cast<uint4*>(sm)[i] = zero;
      int h0 = 0, h1 = 0, p = 0, k0 = 0, k1 = 0;
      if (b >= 0) {
        if (a.r.d_repetition) f.rep = a.r.d_repetition[b];
        if (a.r.d_frequency) f.freq = a.r.d_frequency[b];
        if (a.r.d_presence) f.pres = a.r.d_presence[b];
        if (a.r.d_temperature) f.temp = a.r.d_temperature[b];
        if (!(f.temp > 0.f)) f.temp = 1.f;
        f.rep_inv = 1.f / f.rep;
        f.temp_inv = 1.f / f.temp;
        f.divide = !usual(f.rep) || !usual(f.temp);
        if (a.r.d_hist) {
          h0 = a.r.d_hist_off[b], h1 = a.r.d_hist_off[b + 1];
          p = h0 + (a.r.d_prompt_len ? a.r.d_prompt_len[b] : 0);
        }
        if (biased) k0 = a.r.d_bias_off[b], k1 = a.r.d_bias_off[b + 1];
      }
      __syncthreads();
      // a token's word, and its second one if it lies at a border
      const auto each = [&](int v, auto&& go) {
        if ((unsigned)v >= (unsigned)a.V) return;
        const int rel = v - v0 + held_shift + 8;
        if (rel < 0 || rel >= a.subs * kSub + 16) return;
        const int w = rel / kSub, i = rel % kSub;
        if (w < a.subs) go(w * kRegion + i);
        if (w > 0 && i < 16) go((w - 1) * kRegion + kSub + i);
      };
#pragma unroll 4
      for (int k = h0 + tid; k < h1; k += threads)
        each(__ldg(a.r.d_hist + k), [&](int i) {
          if (k < p) atomicOr(sm + i, kPrompt);
          else atomicAdd(sm + i, 1u);
        });
      for (int k = k0 + tid; k < k1; k += threads)
        each(a.r.d_bias_tok[k], [&](int i) { atomicMax(all_bias + i, (uint32_t)(k - k0) + 1u); });   // (the later entry)
      __syncthreads();
    }
    const int first = 8 + held_shift - shift;   // word of token t0
    const float* bias_val = biased && b >= 0 ? a.r.d_bias_val + a.r.d_bias_off[b] : nullptr;
    const bool path = a.mask && b >= 0 && a.r.d_tree_tok;
    // the row's path: `by` added to the words of its tokens among the warp's
    const auto walk = [&](uint32_t by) {
      const int q0 = __ldg(a.r.d_cu_q + b), len = __ldg(a.r.d_cu_q + b + 1) - q0;
      for (int w = lane; w < a.words && 32 * w < len; w += 32) {
        uint32_t bits = __ldg(a.mask + (long long)row * a.words + w);
        while (bits) {
          const int j = 32 * w + __ffs(bits) - 1;
          bits &= bits - 1;
          if (j >= len) break;
          const int v = __ldg(a.r.d_tree_tok + q0 + j), i = v - t0;
          if (i >= 0 && i < kSub && v >= 0 && v < a.V) atomicAdd(cnt + first + i, by);
        }
      }
      __syncwarp();
    };
    if (path) walk(1u);
    const int s = a.state && a.r.d_grammar ? __ldg(a.state + row) : -1;
    const uint32_t* allowed = s >= 0 && s < a.r.n_states ? a.r.d_grammar + s * a.r.grammar_stride : nullptr;
    const bool straight = (first & 3) == 0;
    const bool wide = (reinterpret_cast<uintptr_t>(out + (long long)t0 * O::SIZE) & 15) == 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = (lane + 32 * u) * N, t = t0 + i;
      if (t + N <= 0 || t >= a.V) continue;
      float x[N];
      uint32_t w[N];
      if (straight) {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
          const uint4 c = *reinterpret_cast<const uint4*>(cnt + first + i + j);
          w[j] = c.x, w[j + 1] = c.y, w[j + 2] = c.z, w[j + 3] = c.w;
        }
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) w[j] = cnt[first + i + j];
      }
      uint32_t any = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        x[j] = I::at(raw[u], j);
        any |= w[j];
      }
      if (any) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          if (!w[j]) continue;
          const uint32_t c = w[j] & ~kPrompt;
          x[j] = x[j] > 0.f ? (f.divide ? x[j] / f.rep : x[j] * f.rep_inv) : x[j] * f.rep;
          if (c) x[j] = x[j] - f.freq * (float)c - f.pres;
        }
      }
      if (bias_val) {
        uint32_t e[N], any_bias = 0;
        if (straight) {
#pragma unroll
          for (int j = 0; j < N; j += 4) {
            const uint4 c = *reinterpret_cast<const uint4*>(bias + first + i + j);
            e[j] = c.x, e[j + 1] = c.y, e[j + 2] = c.z, e[j + 3] = c.w;
          }
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j) e[j] = bias[first + i + j];
        }
#pragma unroll
        for (int j = 0; j < N; ++j) any_bias |= e[j];
        if (any_bias) {
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (e[j]) x[j] += __ldg(bias_val + e[j] - 1);
        }
      }
      if (f.divide) {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = x[j] / f.temp;
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] *= f.temp_inv;
      }
      if (allowed) {
        const int tw = max(t, 0), last = (a.V - 1) >> 5;
        const uint32_t g = __funnelshift_r(__ldg(allowed + (tw >> 5)), __ldg(allowed + min((tw >> 5) + 1, last)), tw & 31);
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (!(g >> (t + j - tw & 31) & 1)) x[j] = -INFINITY;   // (a token before the row is not stored)
      }
      if (t >= 0 && t + N <= a.V && wide) {
        if constexpr (OUT == ATSPEED_F32) {
#pragma unroll
          for (int j = 0; j < N; j += 4)
            __stcs(reinterpret_cast<float4*>(out + ((long long)t + j) * 4), make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]));
        } else {
          constexpr bool H = OUT == ATSPEED_F16;
          *reinterpret_cast<uint4*>(out + (long long)t * O::SIZE) =
              make_uint4(pack2(x[0], x[1], H), pack2(x[2], x[3], H), pack2(x[4], x[5], H), pack2(x[6], x[7], H));
        }
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (t + j >= 0 && t + j < a.V) O::store1(out + (long long)(t + j) * O::SIZE, x[j]);
      }
    }
    if (path) {
      __syncwarp();
      walk(~0u);
    }
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
  // Warps of 1024 tokens (7 more for rows that begin between 16-byte addresses), as evenly over CTAs as they go; rows a CTA:
  // a request's history is counted once for all of them, as long as every SM keeps a few CTAs.
  const int subs = (vocab + 7 + kSub - 1) / kSub, chunks = (subs + kWarps - 1) / kWarps;
  a.subs = (subs + chunks - 1) / chunks;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return ATSPEED_E_CUDA;
  const long long room = 12LL * gemm_grid_size(dev);
  a.rows = (int)std::min(16LL, std::max(1LL, (long long)R * chunks / room));
  const long long groups = (R + a.rows - 1LL) / a.rows;
  if (groups > 65535) return ATSPEED_E_SHAPE;
  const int smem = a.subs * kRegion * 4 * (r.d_bias_off ? 2 : 1);
  const dim3 grid(chunks, (unsigned)groups);
  auto go = [&](auto kernel, std::atomic<unsigned long long>& done) {
    if (smem_attr_once(done, kernel, kWarps * kRegion * 8) != cudaSuccess) return ATSPEED_E_CUDA;
    kernel<<<grid, 32 * a.subs, smem, (cudaStream_t)stream>>>(a);
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
