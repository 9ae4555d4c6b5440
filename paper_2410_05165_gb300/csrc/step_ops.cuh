// Shared by the operators of a batched serving step (plan, cache append, tree attention, logit rules) and those after its logits
// (beam selection, page fork, page copies, token compaction).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "atspeed.h"

namespace atspeed {

constexpr int kMaxRequests = 16384;   // two 32-bit words of shared memory a request in the plan's kernel

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline int dtype_size(int t) { return t == ATSPEED_F32 ? 4 : t == ATSPEED_BF16 || t == ATSPEED_F16 ? 2 : 0; }

// Memory that a call reads or writes (null: none).
struct Span {
  const void* at;
  long long bytes;
  bool meets(const Span& b) const {
    const uintptr_t x = reinterpret_cast<uintptr_t>(at), y = reinterpret_cast<uintptr_t>(b.at);
    return x && y && x < y + b.bytes && y < x + bytes;
  }
};
// Whether an output shares memory with an input or with another output.
template <size_t OUT, size_t IN>
inline bool outputs_overlap(const Span (&out)[OUT], const Span (&in)[IN]) {
  for (size_t i = 0; i < OUT; ++i) {
    for (const Span& s : in)
      if (out[i].meets(s)) return true;
    for (size_t j = 0; j < i; ++j)
      if (out[i].meets(out[j])) return true;
  }
  return false;
}

// Pointers, types and strides of a paged cache (what the operators that read or write it need of it alike).
inline atspeed_status check_pages(const atspeed_kv_pages* c) {
  if (!c || !c->d_k || !c->d_v || c->n_pages <= 0 || c->page_size <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0)
    return ATSPEED_E_ARG;
  const bool types = (c->k_type == ATSPEED_BF16 && (c->v_type == ATSPEED_BF16 || c->v_type == ATSPEED_F16)) ||
                     (c->k_type == ATSPEED_F16 && c->v_type == ATSPEED_F16);
  if (!types || !aligned16(c->d_k) || !aligned16(c->d_v)) return ATSPEED_E_ARG;
  for (int i = 0; i < 3; ++i)
    if (c->k_stride[i] < 0 || c->v_stride[i] < 0 || c->k_stride[i] % 8 || c->v_stride[i] % 8) return ATSPEED_E_ARG;
  return ATSPEED_OK;
}

// The tree attention's error word on the current device (ATSPEED_DEV_ERR_* bits); null if it cannot be found.
unsigned int* tree_attn_err_word();

inline atspeed_status launch_status() { return cudaGetLastError() == cudaSuccess ? ATSPEED_OK : ATSPEED_E_CUDA; }

// Two values rounded to a pair of 16-bit ones.
__device__ __forceinline__ uint32_t pack2(float lo, float hi, bool f16) {
  uint32_t r;
  if (f16)
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint32_t v, bool f16) {
  if (f16) return __half22float2(*reinterpret_cast<const __half2*>(&v));
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

}  // namespace atspeed
