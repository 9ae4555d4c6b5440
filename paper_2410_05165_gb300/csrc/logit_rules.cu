// Penalties, biases, grammar masks and temperature on next-token logits (atspeed_op_adjust_logits).
//   c(v) = occurrences of v in the request's output and on the row's path in its tree, seen(v) = c(v) > 0 or v in the prompt
//   x <- seen ? (x > 0 ? x / rep : x * rep) : x;  x <- x - freq c - pres [c > 0] + bias(v);  forbidden: -inf;  x <- x / temp
// Bound: HBM (each logit read and written once).  A CTA holds one word a token of a vocabulary chunk in shared memory,
// counts the request's history into it once and walks several rows of that request over the chunk, adding each row's path
// before and taking it away after; so the history is scanned once per chunk and group of rows, not once per row.
#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 8192;            // tokens of a chunk
constexpr uint32_t kPrompt = 1u << 31;  // the token occurs in the prompt; below it the count in the output

struct RulesArgs {
  const void* in;
  void* out;
  long long ld_in, ld_out;
  int R, V, n, rows, words;   // rows: consecutive rows a CTA takes
  const int* req;
  const uint32_t* mask;
  const int* state;
  atspeed_logit_rules r;
};

template <int TYPE>
__device__ __forceinline__ float load1(const void* p, long long i) {
  if constexpr (TYPE == ATSPEED_F32) return static_cast<const float*>(p)[i];
  if constexpr (TYPE == ATSPEED_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  return __half2float(static_cast<const __half*>(p)[i]);
}
template <int TYPE>
__device__ __forceinline__ void store1(void* p, long long i, float x) {
  if constexpr (TYPE == ATSPEED_F32) static_cast<float*>(p)[i] = x;
  else if constexpr (TYPE == ATSPEED_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(x);
  else static_cast<__half*>(p)[i] = __float2half_rn(x);
}

template <int IN, int OUT>
__global__ void __launch_bounds__(kThreads) adjust_logits_kernel(const __grid_constant__ RulesArgs a) {
  extern __shared__ uint32_t sm[];
  uint32_t* cnt = sm;                  // [kChunk]
  uint32_t* bias = sm + kChunk;        // [kChunk] index + 1 of the token's bias entry (with biases)
  const int v0 = blockIdx.x * kChunk, nv = min(kChunk, a.V - v0), tid = threadIdx.x;
  const int r0 = blockIdx.y * a.rows, r1 = min(a.R, r0 + a.rows);
  const bool biased = a.r.d_bias_off != nullptr;
  int held = -2;   // the request whose counts the chunk holds
  float rep = 1.f, freq = 0.f, pres = 0.f, temp = 1.f;
  for (int row = r0; row < r1; ++row) {
    int b = a.req[row];
    if (b < 0 || b >= a.n) b = -1;
    if (b != held) {
      __syncthreads();
      for (int i = tid; i < nv; i += kThreads) {
        cnt[i] = 0;
        if (biased) bias[i] = 0;
      }
      __syncthreads();
      rep = 1.f, freq = 0.f, pres = 0.f, temp = 1.f;
      if (b >= 0) {
        if (a.r.d_repetition) rep = a.r.d_repetition[b];
        if (a.r.d_frequency) freq = a.r.d_frequency[b];
        if (a.r.d_presence) pres = a.r.d_presence[b];
        if (a.r.d_temperature) temp = a.r.d_temperature[b];
        if (a.r.d_hist) {
          const int h0 = a.r.d_hist_off[b], h1 = a.r.d_hist_off[b + 1], p = h0 + (a.r.d_prompt_len ? a.r.d_prompt_len[b] : 0);
          for (int k = h0 + tid; k < h1; k += kThreads) {
            const unsigned v = (unsigned)(a.r.d_hist[k] - v0);
            if (v < (unsigned)nv) {
              if (k < p) atomicOr(cnt + v, kPrompt);
              else atomicAdd(cnt + v, 1u);
            }
          }
        }
        if (biased)
          for (int k = a.r.d_bias_off[b] + tid; k < a.r.d_bias_off[b + 1]; k += kThreads) {
            const unsigned v = (unsigned)(a.r.d_bias_tok[k] - v0);
            if (v < (unsigned)nv) atomicMax(bias + v, (uint32_t)k + 1u);   // (the later entry)
          }
      }
      held = b;
      __syncthreads();
    }
    const bool path = a.mask && b >= 0 && a.r.d_tree_tok;
    const auto walk = [&](uint32_t d) {   // the row's path tokens: one more, or one less, each
      const int t0 = a.r.d_cu_q[b], len = a.r.d_cu_q[b + 1] - t0;
      for (int j = tid; j < min(len, 32 * a.words); j += kThreads)
        if (a.mask[(long long)row * a.words + (j >> 5)] >> (j & 31) & 1) {
          const unsigned v = (unsigned)(a.r.d_tree_tok[t0 + j] - v0);
          if (v < (unsigned)nv) atomicAdd(cnt + v, d);
        }
    };
    if (path) {
      walk(1u);
      __syncthreads();
    }
    const int s = a.state && a.r.d_grammar ? a.state[row] : -1;
    const uint32_t* allowed = s >= 0 && s < a.r.n_states ? a.r.d_grammar + s * a.r.grammar_stride : nullptr;
    for (int i = tid; i < nv; i += kThreads) {
      const int v = v0 + i;
      float x = load1<IN>(a.in, row * a.ld_in + v);
      const uint32_t w = cnt[i];
      if (w) {
        x = x > 0.f ? x / rep : x * rep;
        const uint32_t c = w & ~kPrompt;
        if (c) x = x - freq * (float)c - pres;
      }
      if (biased && bias[i]) x += a.r.d_bias_val[bias[i] - 1];
      if (allowed && !(allowed[v >> 5] >> (v & 31) & 1)) x = -INFINITY;
      if (temp > 0.f) x = x / temp;
      store1<OUT>(a.out, row * a.ld_out + v, x);
    }
    if (path) {
      __syncthreads();
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
  a.rows = 8;
  const long long groups = (R + a.rows - 1LL) / a.rows;
  if (groups > 65535) return ATSPEED_E_SHAPE;
  const int smem = kChunk * 4 * (r.d_bias_off ? 2 : 1);
  const dim3 grid((vocab + kChunk - 1) / kChunk, (unsigned)groups);
  auto go = [&](auto kernel, std::atomic<unsigned long long>& done) {
    if (smem_attr_once(done, kernel, kChunk * 8) != cudaSuccess) return ATSPEED_E_CUDA;
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
