// Rotary embedding of new tokens and their entry into a paged cache (atspeed_op_rope_append).
//   a_i = pos * theta^(-2 i / hd);  (x_i, x_(i + hd/2)) -> (x_i cos a_i - x_(i+hd/2) sin a_i, x_(i+hd/2) cos a_i + x_i sin a_i)
// The angle is kept in turns, as a 64-bit fraction of one: f_i = theta^(-2 i / hd) / (2 pi) * 2^64 comes from the host, and
// pos * f_i modulo 2^64 is the turn's fraction, as exact as f_i (2^-53 of it) at any position (a 32-bit pos * freq is off
// by up to 4e-3 radians at position 65 000).  Bound: HBM (2 or 4 bytes a value in, 2 out): 3840 rows of 96
// heads of 128 from 32 bits, 283 MB, take 48 us, 5.9 TB/s.  A row a CTA, eight values a thread and access.
#include <cmath>

#include "common.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxHalf = 128;

struct AppendArgs {
  const void* qkv;
  long long stride, q_stride;
  int T, H, Hkv, hd, page;
  long long rows;                       // cache rows
  const long long* slot;
  const int* pos;
  void *q, *k, *v;
  long long ks[3], vs[3];
  bool src_f16, k_f16, v_f16;
  unsigned long long freq[kMaxHalf];    // turns per position, 2^-64
};

// Eight values from 16-byte aligned memory of type F32 (in 32 bits) or one of the 16-bit ones.
template <bool F32>
__device__ __forceinline__ void load8(const void* p, long long i, bool f16, float (&x)[8]) {
  if constexpr (F32) {
    const float4* s = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
    const float4 a = __ldcs(s), b = __ldcs(s + 1);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
    const uint4 v = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i));
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = unpack2(u[j], f16);
      x[2 * j] = f.x, x[2 * j + 1] = f.y;
    }
  }
}
__device__ __forceinline__ void store8(void* p, long long i, bool f16, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) =
      make_uint4(pack2(x[0], x[1], f16), pack2(x[2], x[3], f16), pack2(x[4], x[5], f16), pack2(x[6], x[7], f16));
}

// One CTA a token; a thread takes eight dimensions i and their partners i + hd/2 of one head at a time.
template <bool F32>
__global__ void __launch_bounds__(kThreads) rope_append_kernel(const __grid_constant__ AppendArgs a) {
  __shared__ float s_cos[kMaxHalf], s_sin[kMaxHalf];
  const int t = blockIdx.x, half = a.hd / 2, chunks = half / 8;
  if (a.pos) {
    const long long pos = a.pos[t];
    for (int i = threadIdx.x; i < half; i += kThreads) {
      const unsigned long long turn = (unsigned long long)pos * a.freq[i];
      // (the fraction of a turn in [-1/2, 1/2), in half turns)
      sincospif((float)(int)(turn >> 32) * 0x1p-31f, &s_sin[i], &s_cos[i]);
    }
    __syncthreads();
  }
  const long long slot = a.slot[t];
  const bool stored = slot >= 0 && slot < a.rows;
  const long long pg = stored ? slot / a.page : 0, row = stored ? slot % a.page : 0;
  const int heads = a.H + 2 * a.Hkv;
  for (int w = threadIdx.x; w < heads * chunks; w += kThreads) {
    const int h = w / chunks, i = (w - h * chunks) * 8;
    if (h >= a.H && !stored) continue;
    const long long src = t * a.stride + (long long)h * a.hd + i;
    float lo[8], hi[8];
    load8<F32>(a.qkv, src, a.src_f16, lo);
    load8<F32>(a.qkv, src + half, a.src_f16, hi);
    if (a.pos && h < a.H + a.Hkv) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float c = s_cos[i + j], s = s_sin[i + j], x = lo[j], y = hi[j];
        lo[j] = x * c - y * s;
        hi[j] = y * c + x * s;
      }
    }
    void* dst;
    long long at;
    bool f16;
    if (h < a.H) {
      dst = a.q, at = t * a.q_stride + (long long)h * a.hd, f16 = a.k_f16;
    } else if (h < a.H + a.Hkv) {
      dst = a.k, at = pg * a.ks[0] + row * a.ks[1] + (h - a.H) * a.ks[2], f16 = a.k_f16;
    } else {
      dst = a.v, at = pg * a.vs[0] + row * a.vs[1] + (h - a.H - a.Hkv) * a.vs[2], f16 = a.v_f16;
    }
    store8(dst, at + i, f16, lo);
    store8(dst, at + i + half, f16, hi);
  }
}

}  // namespace
}  // namespace atspeed

using namespace atspeed;

extern "C" atspeed_status atspeed_op_rope_append(atspeed_stream stream, const void* d_qkv, atspeed_dtype src_type,
                                                 int64_t qkv_stride, int T, int n_heads, const atspeed_kv_pages* cache,
                                                 const int64_t* d_slot, const int32_t* d_pos, float theta, void* d_q,
                                                 int64_t q_stride) {
  const atspeed_status st = check_pages(cache);
  if (st != ATSPEED_OK) return st;
  const atspeed_kv_pages& c = *cache;
  if (!d_qkv || !d_slot || T <= 0 || n_heads < 0 || (n_heads > 0 && !d_q)) return ATSPEED_E_ARG;
  if (src_type != ATSPEED_F32 && src_type != c.k_type) return ATSPEED_E_ARG;
  if (c.head_dim % 16 || c.head_dim > 2 * kMaxHalf) return ATSPEED_E_SHAPE;
  const int64_t width = (int64_t)(n_heads + 2 * (int64_t)c.n_kv_heads) * c.head_dim;
  if (n_heads > 65536 || c.n_kv_heads > 65536) return ATSPEED_E_SHAPE;
  const int per16 = 16 / dtype_size(src_type);
  if (qkv_stride < width || qkv_stride % per16 || !aligned16(d_qkv)) return ATSPEED_E_ARG;
  if (n_heads > 0 && (q_stride < (int64_t)n_heads * c.head_dim || q_stride % 8 || !aligned16(d_q))) return ATSPEED_E_ARG;
  if (d_pos && !(theta > 0.f && std::isfinite(theta))) return ATSPEED_E_ARG;
  AppendArgs a = {};
  a.qkv = d_qkv, a.stride = qkv_stride, a.q_stride = q_stride;
  a.T = T, a.H = n_heads, a.Hkv = c.n_kv_heads, a.hd = c.head_dim, a.page = c.page_size;
  a.rows = (long long)c.n_pages * c.page_size;
  a.slot = reinterpret_cast<const long long*>(d_slot), a.pos = d_pos;
  a.q = d_q, a.k = c.d_k, a.v = c.d_v;
  for (int i = 0; i < 3; ++i) a.ks[i] = c.k_stride[i], a.vs[i] = c.v_stride[i];
  a.src_f16 = src_type == ATSPEED_F16, a.k_f16 = c.k_type == ATSPEED_F16, a.v_f16 = c.v_type == ATSPEED_F16;
  if (d_pos)
    for (int i = 0; i < c.head_dim / 2; ++i) {
      const double turns = std::pow((double)theta, -2.0 * i / c.head_dim) * 0.15915494309189535;   // 1 / (2 pi)
      a.freq[i] = (unsigned long long)((turns - std::floor(turns)) * 0x1p64);   // (whole turns drop out: theta < 1)
    }
  if (src_type == ATSPEED_F32)
    rope_append_kernel<true><<<T, kThreads, 0, (cudaStream_t)stream>>>(a);
  else
    rope_append_kernel<false><<<T, kThreads, 0, (cudaStream_t)stream>>>(a);
  return launch_status();
}
