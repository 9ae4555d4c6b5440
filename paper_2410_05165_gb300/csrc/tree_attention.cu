// Attention of new tokens (trees, chains) over a batch's paged caches (atspeed_op_tree_attention), on the tensor cores.
//   o = sum_j w_j v_j / sum_j w_j, w_j = exp(scale q.k_j), over the positions j < ctx and those of the token's ancestors
//
// The rows of a (request, key head) are its new tokens times the G query heads that share the key head: they read the same
// K and V, so a block of up to 256 rows reads each K / V tile of 128 keys once.  A tile is two products on tcgen05 with M =
// 128 rows: S = Q K^T (both K-major in shared memory) into TMEM, and O += P V with P (16 bits) as TMEM operand over S's
// columns and V in place, MN-major.  One thread a row runs the softmax from TMEM: no shuffles, no shared memory; O is scaled
// only where the running maximum rises by more than 2^8 (all weights are relative to the maximum in use, so the quotient
// is the same).
//
// Two streams of (S, P, O) alternate on the tensor core, each with a warpgroup of its own: one's softmax runs under the
// other's products.  Blocks of more than 128 rows: a stream is 128 of the rows, each sees every tile.  Fewer: both hold the
// same rows and take alternate tiles; they are joined at the end.  (Padding a single token's G rows to 128 costs tensor
// time that the tile's 64 KB of K and V, 2800 clocks of an SM's share of the HBM, leave free: 1024 clocks.)
//
// Work is the concatenation of all blocks' tiles, cut into one equal range a CTA (every CTA finds its own range from the
// lengths); a block cut by a range's end is summed from partial results in device memory, each of its CTAs taking a share
// of the rows, in range order.  Waits for partial results come after all own results are out and the grid is launched
// cooperatively, so that they end; they are bounded all the same.
//
// Roles (384 threads): warp 0 copies (TMA), warp 1 issues the products, warps 2-3 load Q, warps 4-7 and 8-11 are the streams.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <cmath>

#include "common.cuh"
#include "gemm.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

__device__ unsigned int g_tree_attn_err;

constexpr int kThreads = 384;
constexpr int kTile = 128;       // keys of a tile
constexpr int kBlock = 256;      // rows of a block
constexpr int kRoleRegs = 80, kStreamRegs = 208;
static_assert(128 * kRoleRegs + 256 * kStreamRegs <= kThreads * 168, "registers at launch");
constexpr float kSlack = 8.f;    // rise of the running maximum (log2) below which O keeps its scale
constexpr int kMaxCtas = 512;    // counters in the workspace

template <int HD>
struct Cfg {
  static constexpr int SW = HD >= 64 ? 128 : 64;       // bytes of a panel's row, and its swizzle
  static constexpr int PANELS = HD * 2 / SW;
  static constexpr int PANEL = kTile * SW;
  static constexpr int TILE = PANELS * PANEL;          // K or V tile, or 128 rows of Q
  static constexpr int STAGES = HD == 128 ? 5 : 8;
  static constexpr int Q_OFF = STAGES * TILE;
  static constexpr int X_OFF = Q_OFF + 2 * TILE;       // (m, l) of both streams
  static constexpr int BAR_OFF = X_OFF + 2 * 128 * 8;
  static constexpr int SMEM = BAR_OFF + 512;
  static constexpr int S_COL = 128, O_COL = 256;       // TMEM columns: S / P of stream s at s * 128, O at 256 + s * HD
  static constexpr int O_STEP = HD;
  static constexpr size_t PART = (size_t)kBlock * (HD + 2) * 4;   // bytes of a partial result: O [256][HD], (m, l) [256]
};
static_assert(Cfg<128>::SMEM <= 232448 && Cfg<64>::SMEM <= 232448, "shared memory of a CTA");

struct TreeAttnArgs {
  const uint16_t *q, *v;
  long long vs[3], q_stride, out_stride;
  int H, Hkv, G, n, T, page, width, words, cap;   // cap: positions that a table row covers
  const int *cu_q, *ctx, *table;
  const uint32_t* mask;
  float c;                                        // scale * log2(e)
  uint16_t* out;
  float* lse;
  bool k_f16, v_f16;
  unsigned char* parts;
  int* arrived;                                   // [kMaxCtas] partial results of the block that starts in a CTA
  int* done;                                      // [kMaxCtas] shares of it that are merged
  unsigned int* err;
};

// ---------------------------------------------------------------------------------------------
// the walk over (request, key head, block): every role does it for itself
// ---------------------------------------------------------------------------------------------
struct Request {
  int q, ctx, t0, rows, blocks;
};
__device__ __forceinline__ Request request(const TreeAttnArgs& a, int b) {
  Request r;
  r.t0 = __ldg(a.cu_q + b);
  r.q = __ldg(a.cu_q + b + 1) - r.t0;
  r.ctx = __ldg(a.ctx + b);
  // (offsets outside the call's rows: nothing of the request is read or written)
  if (r.t0 < 0 || r.q < 0 || r.t0 > a.T - r.q) r.q = 0;
  r.rows = r.q * a.G;
  r.blocks = r.ctx < 0 ? 0 : (r.rows + kBlock - 1) / kBlock;
  return r;
}
__device__ __forceinline__ int block_keys(const TreeAttnArgs& a, const Request& r, int blk) {
  const int last = a.mask ? r.q : (min(r.rows, (blk + 1) * kBlock) - 1) / a.G + 1;
  return (int)min((long long)r.ctx + last, (long long)a.cap);
}
__device__ __forceinline__ int tiles_of(int keys) { return (keys + kTile - 1) / kTile; }
__device__ __forceinline__ long long request_units(const TreeAttnArgs& a, const Request& r) {
  if (r.blocks == 0) return 0;
  long long u = 0;
  if (a.mask) u = (long long)r.blocks * tiles_of(block_keys(a, r, 0));
  else
    for (int i = 0; i < r.blocks; ++i) u += tiles_of(block_keys(a, r, i));
  return u * a.Hkv;
}

struct Start {      // a CTA's range: where it begins
  long long u0, u1, units;
  int b, kh, blk, tile, ctas;
};

struct Walk {
  const TreeAttnArgs& a;
  Request r;
  long long left;     // units of the range from this block on
  int b, kh, blk;
  int tile0, tiles;   // this CTA's tiles of the block
  int all, keys;      // tiles and keys of the whole block
  __device__ Walk(const TreeAttnArgs& args, const Start& s) : a(args), left(s.u1 - s.u0), b(s.b), kh(s.kh), blk(s.blk) {
    if (left <= 0) return;
    r = request(a, b);
    block(s.tile);
  }
  __device__ void block(int first) {
    keys = block_keys(a, r, blk);
    all = tiles_of(keys);
    tile0 = first;
    tiles = (int)min((long long)(all - first), left);
  }
  __device__ bool more() const { return left > 0; }
  __device__ void next() {
    left -= tiles;
    if (left <= 0) return;
    if (++blk == r.blocks) {
      blk = 0;
      if (++kh == a.Hkv) {
        kh = 0;
        do r = request(a, ++b);
        while (r.blocks == 0 && b < a.n - 1);
      }
    }
    block(0);
  }
  __device__ int rows() const { return min(kBlock, r.rows - blk * kBlock); }
  __device__ bool dual() const { return rows() > 128; }
};

// ---------------------------------------------------------------------------------------------
// instructions
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
          smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void mma_ss(uint32_t lead, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n .reg .pred e, p;\n setp.ne.b32 e, %5, 0;\n setp.ne.b32 p, %4, 0;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(add), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t lead, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n .reg .pred e, p;\n setp.ne.b32 e, %5, 0;\n setp.ne.b32 p, %4, 0;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(add), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void tmem_st_32x32b_x32(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
      "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]),
      "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]),
      "r"(v[31])
      : "memory");
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Shared-memory descriptors (fields: common.cuh, smem_desc_sw128).  stride: between groups of eight rows of a panel; lead:
// between panels of an MN-major operand wider than one.  Layout 2 is the 128-byte swizzle, 4 the 64-byte one.
template <int SW>
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t lead) {
  return (uint64_t)((addr >> 4) & 0x3FFFu) | (uint64_t)((lead >> 4) & 0x3FFFu) << 16 | (uint64_t)((8u * SW) >> 4) << 32 |
         (uint64_t)1u << 46 | (uint64_t)(SW == 128 ? 2u : 4u) << 61;
}
// Instruction descriptor (fields: idesc_bf16_f32); bit 16: B is MN-major
__device__ __forceinline__ uint32_t instr_desc(int n, bool f16, bool b_mn) {
  const uint32_t t = f16 ? 0u : 1u;
  return (1u << 4) | (t << 7) | (t << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}

// Place of a K or V tile in the order of the copies: blocks on both streams' rows read K, V, K, V, ..; blocks that
// alternate tiles read K one ahead (K0, K1, V0, K2, V1, ..), as the products do.
__device__ __forceinline__ int seq_k(bool dual, int i) { return dual ? 2 * i : max(0, 2 * i - 1); }
__device__ __forceinline__ int seq_v(bool dual, int i, int n) { return dual ? 2 * i + 1 : min(2 * i + 2, 2 * n - 1); }

__device__ __forceinline__ bool finite16(uint32_t two, bool f16, uint32_t& clean) {
  const uint32_t e = f16 ? 0x7c00u : 0x7f80u;
  clean = two;
  if ((two & e) == e) clean &= 0xffff0000u;
  if ((two >> 16 & e) == e) clean &= 0x0000ffffu;
  return clean == two;
}

// 32 bits of a row's mask from bit j0 on (bits outside [0, q) are 0)
__device__ __forceinline__ uint32_t mask_window(const uint32_t* row, int words, int j0, int q) {
  const auto word = [&](int i) { return i >= 0 && i < words ? __ldg(row + i) : 0u; };
  const int w = j0 >> 5, sh = j0 & 31;   // (arithmetic: j0 may be negative)
  const uint32_t x = __funnelshift_r(word(w), word(w + 1), sh);
  const int up = q - j0;
  return up >= 32 ? x : up <= 0 ? 0u : x & ((1u << up) - 1u);
}
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// The 32 keys from `key` on that row token i of request r sees.
__device__ __forceinline__ uint32_t seen_word(const TreeAttnArgs& a, const Request& r, int i, int key) {
  const int j0 = key - r.ctx;
  uint32_t x = a.mask ? mask_window(a.mask + (long long)(r.t0 + i) * a.words, a.words, j0, r.q) : low_bits(i + 1 - j0);
  x |= low_bits(-j0);                    // cached positions
  return x & low_bits(a.cap - key);
}

// ---------------------------------------------------------------------------------------------
// a partial result's place, and the block's CTAs
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ int cta_of(long long u, const Start& s) { return (int)(((u + 1) * s.ctas - 1) / s.units); }

template <int HD>
__device__ __forceinline__ float* part_of(const TreeAttnArgs& a, int cta, int slot) {
  return reinterpret_cast<float*>(a.parts + (size_t)(2 * cta + slot) * Cfg<HD>::PART);
}

// Four columns of a row: sum over a block's partial results in their order.
template <int HD>
__device__ __forceinline__ void merge_share(const TreeAttnArgs& a, const Request& r, int kh, int blk, int first, int parts,
                                            int share, int tid) {
  constexpr int V4 = HD / 4;
  const int rows = min(kBlock, r.rows - blk * kBlock), total = rows * V4;
  const int i0 = (int)((long long)total * share / parts), i1 = (int)((long long)total * (share + 1) / parts);
  for (int i = i0 + tid; i < i1; i += 256) {
    const int row = i / V4, c4 = i % V4;
    const auto ml = [&](int p) {
      return __ldcg(reinterpret_cast<const float2*>(part_of<HD>(a, first + p, p == 0) + kBlock * HD) + row);
    };
    float m = -INFINITY;
    for (int p = 0; p < parts; ++p) m = fmaxf(m, ml(p).x);
    float l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
      const float2 x = ml(p);
      const float4 y = __ldcg(reinterpret_cast<const float4*>(part_of<HD>(a, first + p, p == 0) + row * HD) + c4);
      // (a part that saw none of the row's keys has l = 0 and no scale; a NaN in l stays one)
      const float w = x.x == -INFINITY ? x.y : exp2_fast(x.x - m);
      l += x.x == -INFINITY ? x.y : w * x.y;
      o.x += w * y.x, o.y += w * y.y, o.z += w * y.z, o.w += w * y.w;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int rg = blk * kBlock + row, t = r.t0 + rg / a.G, h = kh * a.G + rg % a.G;
    uint2 u = make_uint2(pack2(o.x * inv, o.y * inv, a.k_f16), pack2(o.z * inv, o.w * inv, a.k_f16));
    *reinterpret_cast<uint2*>(a.out + (long long)t * a.out_stride + (long long)h * HD + c4 * 4) = u;
    if (a.lse && c4 == 0) a.lse[(long long)t * a.H + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
  }
}

__device__ __forceinline__ bool wait_count(const int* p, int want, unsigned int* err) {
  const unsigned long long t0 = globaltimer_ns();
  for (unsigned it = 1;; ++it) {
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    if (v >= want) return true;
    if ((it & 255u) == 0u && globaltimer_ns() - t0 > kWaitBudgetNs) {
      set_error(err, ATSPEED_DEV_ERR_TIMEOUT);
      return false;
    }
  }
}

// A wait of a whole warp, which goes on together; after the first that gave up the rest are not waited for (the loops run
// to their ends without the work, so that every barrier meets its threads).
__device__ __forceinline__ bool warp_wait(bool ok, uint64_t* bar, uint32_t parity, unsigned int* err) {
  if (ok) ok = mbar_wait(bar, parity, err);
  return __all_sync(0xffffffffu, ok);
}

template <int HD>
__global__ void __launch_bounds__(kThreads, 1)
    tree_attention_kernel(const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv,
                          const __grid_constant__ TreeAttnArgs a) {
  using C = Cfg<HD>;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::BAR_OFF);
  uint64_t* empty = full + C::STAGES;
  uint64_t* s_full = empty + C::STAGES;   // [2] S of a stream is in TMEM
  uint64_t* p_ready = s_full + 2;         // [2] P of a stream is in TMEM
  uint64_t* q_full = p_ready + 2;
  uint64_t* q_free = q_full + 1;
  uint64_t* o_done = q_free + 1;          // the block's products are complete
  uint64_t* o_free = o_done + 1;          // its O is read
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_free + 1);
  volatile int* odd_v = reinterpret_cast<int*>(tmem_slot + 1);   // a NaN or infinity was found in a new token's V
  Start* start = reinterpret_cast<Start*>(smem + C::BAR_OFF + 256);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned int* err = a.err;

  // ---- this CTA's range of the call's units ----
  {
    long long* sums = reinterpret_cast<long long*>(smem);   // (the ring is not in use yet)
    const int per = (a.n + kThreads - 1) / kThreads, b0 = min(a.n, tid * per), b1 = min(a.n, b0 + per);
    long long own = 0;
    for (int b = b0; b < b1; ++b) own += request_units(a, request(a, b));
    long long sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += x;
    }
    if (lane == 31) sums[warp] = sum;
    if (warp == 2) tmem_alloc(tmem_slot, 512);
    if (tid == 0) {
      for (int i = 0; i < C::STAGES; ++i) mbar_init(full + i, 1), mbar_init(empty + i, 1);
      for (int i = 0; i < 2; ++i) mbar_init(s_full + i, 1), mbar_init(p_ready + i, 4);
      mbar_init(q_full, 2);
      mbar_init(q_free, 1);
      mbar_init(o_done, 1);
      mbar_init(o_free, 8);
      fence_mbar_init();
      *odd_v = 0;
      start->u0 = start->u1 = 0;
    }
    if (tid == 32) tma_prefetch_desc(&tmk), tma_prefetch_desc(&tmv);
    __syncthreads();
    long long total = 0, before = sum - own;
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) before += sums[w];
      total += sums[w];
    }
    const int ctas = (int)min((long long)gridDim.x, total), cta = blockIdx.x;
    if (cta < ctas) {
      const long long u0 = cta * total / ctas, u1 = (cta + 1LL) * total / ctas;
      if (u0 >= before && u0 < before + own) {
        int b = b0;
        long long off = u0 - before;
        for (;; ++b) {
          const Request r = request(a, b);
          const long long u = request_units(a, r);
          if (off < u) {
            const long long head = u / a.Hkv;
            int blk = 0;
            start->kh = (int)(off / head);
            off %= head;
            for (int k; off >= (k = tiles_of(block_keys(a, r, blk))); ++blk) off -= k;
            start->blk = blk;
            break;
          }
          off -= u;
        }
        start->b = b;
        start->tile = (int)off;
        start->u0 = u0, start->u1 = u1, start->units = total, start->ctas = ctas;
      }
    }
    // requests that were not served: zeros
    for (int b = blockIdx.x; b < a.n; b += gridDim.x) {
      const Request r = request(a, b);
      if (r.ctx >= 0) continue;
      for (long long i = tid; i < (long long)r.rows * a.Hkv; i += kThreads) {
        const int t = r.t0 + (int)(i / a.H), h = (int)(i % a.H);
        uint4* o = reinterpret_cast<uint4*>(a.out + (long long)t * a.out_stride + (long long)h * HD);
        for (int k = 0; k < HD / 8; ++k) o[k] = make_uint4(0, 0, 0, 0);
        if (a.lse) a.lse[(long long)t * a.H + h] = -INFINITY;
      }
    }
    fence_proxy_async_shared();   // (the sums were read before copies overwrite them)
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
  }
  const uint32_t tmem = *tmem_slot;
  const Start st = *start;
  bool ok = true;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRoleRegs));
    if (warp == 0) {
      // ---- copies ----
      const int box = min(a.page, kTile), n_box = kTile / box;   // pages (or the half page) of a tile
      const int lp = lane / C::PANELS, panel = lane % C::PANELS;
      unsigned seq = 0;
      for (Walk w(a, st); w.more(); w.next()) {
        const bool dual = w.dual();
        const int n = w.tiles;
        const int* table = a.table + (long long)w.b * a.width;
        const auto pages = [&](int i) {   // this lane's page of tile i (its keys' first position / page)
          const int key = (w.tile0 + i) * kTile + lp * box;
          return i < n && lp < n_box && key < w.keys ? __ldg(table + key / a.page) : 0;
        };
        const auto copy = [&](const CUtensorMap* map, int i, int id) {
          const int slot = seq % C::STAGES;
          ok = warp_wait(ok, empty + slot, (seq / C::STAGES & 1) ^ 1, err);
          ++seq;
          if (!ok) return;
          const int key0 = (w.tile0 + i) * kTile, boxes = min(n_box, (w.keys - key0 + box - 1) / box);
          if (lane == 0) mbar_arrive_expect_tx(full + slot, boxes * box * HD * 2);
          __syncwarp();
          if (lp < boxes)
            tma_load_4d(smem + slot * C::TILE + panel * C::PANEL + lp * box * C::SW, map, full + slot, panel * (C::SW / 2),
                        (key0 + lp * box) % a.page, w.kh, id);
        };
        int ids = pages(0), next = pages(1);
        if (dual) {
          for (int i = 0; i < n; ++i) {
            copy(&tmk, i, ids);
            copy(&tmv, i, ids);
            ids = next;
            next = pages(i + 2);
          }
        } else {
          int last = 0;
          for (int i = 0; i <= n; ++i) {
            if (i < n) copy(&tmk, i, ids);
            if (i > 0) copy(&tmv, i - 1, last);
            last = ids;
            ids = next;
            next = pages(i + 2);
          }
        }
      }
    } else if (warp == 1) {
      // ---- products ----
      const uint32_t lead = elect_one();
      const uint32_t id_s = instr_desc(kTile, a.k_f16, false), id_o = instr_desc(HD, a.v_f16, true);
      unsigned seq0 = 0, item = 0, used[2] = {0, 0};   // used: P's consumed on a stream
      const uint32_t ring = smem_u32(smem), qs = smem_u32(smem + C::Q_OFF);
      for (Walk w(a, st); w.more(); w.next(), ++item) {
        const bool dual = w.dual();
        const int n = w.tiles, steps = dual ? 2 * n : n;
        ok = warp_wait(ok, q_full, item & 1, err);
        const auto scores = [&](int t) {
          const int s = t & 1, i = dual ? t >> 1 : t;
          const unsigned seq = seq0 + seq_k(dual, i), slot = seq % C::STAGES;
          ok = warp_wait(ok, full + slot, seq / C::STAGES & 1, err);
          if (!ok) return;
          tc_fence_after();
          const uint64_t qd = operand_desc<C::SW>(qs + (dual ? s * C::TILE : 0), 16);
          const uint64_t kd = operand_desc<C::SW>(ring + slot * C::TILE, 16);
#pragma unroll
          for (int k = 0; k < HD / 16; ++k) {
            const uint64_t step = (uint64_t)((k * 32 / C::SW) * C::PANEL + k * 32 % C::SW) >> 4;
            mma_ss(lead, tmem + s * C::S_COL, qd + step, kd + step, id_s, k > 0);
          }
          tc_commit_lead(lead, s_full + s);
          if (!dual || s) tc_commit_lead(lead, empty + slot);
          if (t == steps - 1) tc_commit_lead(lead, q_free);
        };
        scores(0);
        if (steps > 1) scores(1);
        ok = warp_wait(ok, o_free, (item & 1) ^ 1, err);
        for (int t = 0; t < steps; ++t) {
          const int s = t & 1, i = dual ? t >> 1 : t;
          const unsigned seq = seq0 + seq_v(dual, i, n), slot = seq % C::STAGES;
          ok = warp_wait(ok, full + slot, seq / C::STAGES & 1, err);
          ok = warp_wait(ok, p_ready + s, used[s] & 1, err);
          ++used[s];
          if (ok) {
            tc_fence_after();
            const uint64_t vd = operand_desc<C::SW>(ring + slot * C::TILE, C::PANEL);
#pragma unroll
            for (int k = 0; k < kTile / 16; ++k)
              mma_ts(lead, tmem + C::O_COL + s * C::O_STEP, tmem + s * C::S_COL + k * 8, vd + (k * 16 * C::SW >> 4), id_o,
                     t > 1 || k > 0);
            if (!dual || s) tc_commit_lead(lead, empty + slot);
            if (t == steps - 1) tc_commit_lead(lead, o_done);
          }
          if (t + 2 < steps) scores(t + 2);
        }
        seq0 += 2 * n;
      }
    } else {
      // ---- Q ----
      const int l64 = tid - 64;
      unsigned item = 0;
      for (Walk w(a, st); w.more(); w.next(), ++item) {
        ok = warp_wait(ok, q_free, (item & 1) ^ 1, err);
        constexpr int CH = HD / 8, U = 8;   // 16-byte chunks of a row, loads in flight
        const int total = w.rows() * CH;
        for (int c0 = l64; c0 < total; c0 += 64 * U) {
          uint4 v[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int ch = c0 + 64 * u;
            if (ch >= total) break;
            const int rg = w.blk * kBlock + ch / CH, t = w.r.t0 + rg / a.G, h = w.kh * a.G + rg % a.G;
            v[u] = __ldg(reinterpret_cast<const uint4*>(a.q + (long long)t * a.q_stride + (long long)h * HD) + ch % CH);
          }
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int ch = c0 + 64 * u;
            if (ch >= total) break;
            const int row = ch / CH, r = row & 127, x = ch % CH, pc = C::SW / 16;   // (pc: chunks of a panel's row)
            const int sw = C::SW == 128 ? r & 7 : (r >> 1) & 3;
            *reinterpret_cast<uint4*>(smem + C::Q_OFF + (row >> 7) * C::TILE + (x / pc) * C::PANEL + r * C::SW +
                                      ((x % pc ^ sw) << 4)) = v[u];
          }
        }
        fence_proxy_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kStreamRegs));
    // ---- a stream: softmax, and the block's results ----
    const int s = (warp - 4) >> 2, r = tid & 127;
    const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);   // this warp's 32 TMEM lanes
    const uint32_t t_s = lanes + s * C::S_COL, t_o = lanes + C::O_COL + s * C::O_STEP;
    float2* xchg = reinterpret_cast<float2*>(smem + C::X_OFF);
    unsigned item = 0, steps_done = 0, seq0 = 0;
    struct Shared {   // a block that other CTAs have a part of
      int b, kh, blk, first, parts;
    } cut[2];
    int cuts = 0;
    long long unit = st.u0;
    for (Walk w(a, st); w.more(); w.next(), ++item) {
      const bool dual = w.dual();
      const int n = w.tiles, rows = w.rows(), row = dual ? s * 128 + r : r;
      const bool mine = row < rows;                              // this thread's row exists
      const bool active = (row & ~31) < rows;                    // .. one of the warp's does
      const int tok = min(w.blk * kBlock + row, w.r.rows - 1) / a.G;
      const int seen_all = min(w.r.ctx, a.cap);                  // keys before this one are seen by every row
      float m = -INFINITY, l = 0.f;
      bool first_step = true;
      for (int i = dual ? 0 : s; i < n; i += dual ? 1 : 2) {
        ok = warp_wait(ok, s_full + s, steps_done & 1, err);
        ++steps_done;
        tc_fence_after();
        const int key0 = (w.tile0 + i) * kTile;
        const bool masked = key0 + kTile > seen_all;
        if (active && ok) {
          uint32_t x[128];
#pragma unroll
          for (int k = 0; k < 4; ++k) tmem_ld_32x32b_x32(t_s + 32 * k, *reinterpret_cast<uint32_t(*)[32]>(x + 32 * k));
          tmem_ld_wait();
          if (masked) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t see = mine ? seen_word(a, w.r, tok, key0 + 32 * k) : 0u;
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (!(see >> j & 1)) x[32 * k + j] = 0xff800000u;   // -infinity
            }
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int j = 0; j < 128; ++j) mx[j & 3] = fmaxf(mx[j & 3], __uint_as_float(x[j]));
          const float m_new = fmaxf(m, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.c);
          const bool rise = mine && (m == -INFINITY ? m_new > m : m_new > m + kSlack);
          if (__any_sync(0xffffffffu, rise)) {
            const float f = !rise ? 1.f : m == -INFINITY ? 0.f : exp2_fast(m - m_new);
            if (!first_step) {
#pragma unroll 1
              for (int k = 0; k < HD; k += 16) {
                uint32_t o[16];
                tmem_ld_32x32b_x16(t_o + k, o);
                tmem_ld_wait();
                float y[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) y[j] = __uint_as_float(o[j]) * f;
                tmem_st_32x32b_x16(t_o + k, y);
              }
            }
            l *= f;
            if (rise) m = m_new;
          }
          const float base = m == -INFINITY ? 0.f : m;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t p[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              const float y0 = exp2_fast(fmaf(__uint_as_float(x[64 * h + 2 * j]), a.c, -base));
              const float y1 = exp2_fast(fmaf(__uint_as_float(x[64 * h + 2 * j + 1]), a.c, -base));
              sum[j & 3] += y0 + y1;
              p[j] = pack2(y0, y1, a.v_f16);
            }
            tmem_st_32x32b_x32(t_s + 32 * h, p);
          }
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
          tmem_st_wait();
        }
        first_step = false;
        if (masked) {
          // V rows that some row of the block does not see: a NaN or infinity there would reach it as 0 x NaN.  They
          // become 0 in the tile (every one of them), and the rows that do see one get it back at the end.
          const unsigned seq = seq0 + seq_v(dual, i, n), slot = seq % C::STAGES;
          ok = warp_wait(ok, full + slot, seq / C::STAGES & 1, err);
          const int first = max(0, seen_all - key0), last = w.keys - key0;
          constexpr int RC = C::SW / 16;
          if (ok)
            for (int k = r; k < (kTile - first) * RC * C::PANELS; k += 128) {
              const int panel = k / ((kTile - first) * RC), at = k % ((kTile - first) * RC);
              uint4* p = reinterpret_cast<uint4*>(smem + slot * C::TILE + panel * C::PANEL + first * C::SW) + at;
              const uint4 v = *p;
              uint4 c;
              const bool f0 = finite16(v.x, a.v_f16, c.x), f1 = finite16(v.y, a.v_f16, c.y);
              const bool f2 = finite16(v.z, a.v_f16, c.z), f3 = finite16(v.w, a.v_f16, c.w);
              if (!(f0 && f1 && f2 && f3)) {
                if (first + at / RC < last) {
                  *odd_v = 1;
                  __threadfence_block();
                }
                *p = c;
              }
            }
          fence_proxy_async_shared();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready + s);
      }
      // ---- the block's (or this part's) result ----
      ok = warp_wait(ok, o_done, item & 1, err);
      tc_fence_after();
      float f0 = 1.f, f1 = 0.f, m_all = m, l_all = l;   // weights of the own rows' O, or of both streams' O
      if (!dual) {
        xchg[s * 128 + r] = make_float2(m, l);
        named_bar_sync(1, 256);
        const float2 e0 = xchg[r], e1 = xchg[128 + r];
        named_bar_sync(1, 256);
        m_all = fmaxf(e0.x, e1.x);
        f0 = e0.x == -INFINITY ? e0.y : exp2_fast(e0.x - m_all);   // (nothing seen: 0, or a NaN)
        f1 = e1.x == -INFINITY ? e1.y : exp2_fast(e1.x - m_all);
        l_all = (e0.x == -INFINITY ? e0.y : f0 * e0.y) + (e1.x == -INFINITY ? e1.y : f1 * e1.y);
      }
      const bool whole = w.tile0 == 0 && n == w.all;
      const int slot = w.tile0 > 0 ? 0 : 1;
      float* part = part_of<HD>(a, blockIdx.x, slot);
      const float inv = whole ? (l_all == 0.f ? 0.f : 1.f / l_all) : 1.f;
      const int rg = w.blk * kBlock + row, t = w.r.t0 + tok, head = w.kh * a.G + (mine ? rg % a.G : 0);
      const int c0 = dual || s == 0 ? 0 : HD / 2, c1 = dual || s == 1 ? HD : HD / 2;
      if (active && ok) {
        const uint32_t o0 = lanes + C::O_COL + (dual ? s * C::O_STEP : 0), o1 = lanes + C::O_COL + C::O_STEP;
#pragma unroll 1
        for (int c = c0; c < c1; c += 16) {
          uint32_t y0[16], y1[16];
          float y[16];
          tmem_ld_32x32b_x16(o0 + c, y0);
          if (!dual) tmem_ld_32x32b_x16(o1 + c, y1);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            y[j] = f0 == 0.f ? 0.f : __uint_as_float(y0[j]) * f0;   // (a stream without tiles leaves its O as it was)
            if (!dual && f1 != 0.f) y[j] += __uint_as_float(y1[j]) * f1;
          }
          if (mine && *odd_v)
            for (int p = max(w.tile0 * kTile, seen_all); p < min(w.keys, (w.tile0 + n) * kTile); ++p) {
              if (!(seen_word(a, w.r, tok, p) & 1)) continue;
              const int id = a.table[(long long)w.b * a.width + p / a.page];
              const uint16_t* v = a.v + id * a.vs[0] + (p % a.page) * a.vs[1] + w.kh * a.vs[2] + c;
              for (int j = 0; j < 16; ++j) {
                uint32_t clean;
                if (!finite16(v[j], a.v_f16, clean)) y[j] += unpack2(v[j], a.v_f16).x;
              }
            }
          if (!mine) continue;
          if (whole) {
            uint4* d = reinterpret_cast<uint4*>(a.out + (long long)t * a.out_stride + (long long)head * HD + c);
#pragma unroll
            for (int j = 0; j < 16; j += 8)
              d[j / 8] = make_uint4(pack2(y[j] * inv, y[j + 1] * inv, a.k_f16), pack2(y[j + 2] * inv, y[j + 3] * inv, a.k_f16),
                                    pack2(y[j + 4] * inv, y[j + 5] * inv, a.k_f16), pack2(y[j + 6] * inv, y[j + 7] * inv, a.k_f16));
          } else {
            float4* d = reinterpret_cast<float4*>(part + row * HD + c);
#pragma unroll
            for (int j = 0; j < 16; j += 4) d[j / 4] = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
          }
        }
        if (mine && (dual || s == 0)) {
          if (!whole) reinterpret_cast<float2*>(part + kBlock * HD)[row] = make_float2(m_all, l_all);
          else if (a.lse)
            a.lse[(long long)t * a.H + head] = l_all == 0.f ? -INFINITY : (m_all + log2f(l_all)) * 0.6931471805599453f;
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_free);
      if (!whole) {
        const long long begin = unit - w.tile0;   // the block's first unit
        Shared& x = cut[cuts++];
        x.b = w.b, x.kh = w.kh, x.blk = w.blk, x.first = cta_of(begin, st);
        x.parts = cta_of(begin + w.all - 1, st) - x.first + 1;
        __threadfence();
        named_bar_sync(2 + s, 128);
        if (r == 0 && ok) asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(a.arrived + x.first) : "memory");
      }
      seq0 += 2 * n;
      unit += n;
    }
    // ---- shares of the blocks that were cut ----
    for (int k = 0; k < cuts; ++k) {
      const Shared x = cut[k];
      if (ok) ok = wait_count(a.arrived + x.first, 2 * x.parts, err);
      ok = named_bar_and(2 + s, 128, ok);
      if (ok) merge_share<HD>(a, request(a, x.b), x.kh, x.blk, x.first, x.parts, blockIdx.x - x.first, s * 128 + r);
      named_bar_sync(2 + s, 128);
      if (r == 0 && ok && atomicAdd(a.done + x.first, 1) == 2 * x.parts - 1) {   // the last share: counters back to zero
        a.arrived[x.first] = 0;
        a.done[x.first] = 0;
      }
    }
  }
  const bool failed = __syncthreads_or(!ok);
  if (failed) {   // copies and products in flight end before the memory goes
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < kDrainNs) {
    }
  }
  tc_fence_after();
  if (warp == 2) {
    tmem_relinquish();
    tmem_dealloc(tmem, 512);
  }
}

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  }();
  return fn;
}

// [page][token][head][dimension] with any strides: boxes of up to 64 dimensions of the tokens of a page (or half of one).
atspeed_status page_map(CUtensorMap* m, const void* base, int type, const atspeed_kv_pages& c, const int64_t* stride) {
  auto fn = encode_fn();
  if (!fn) return ATSPEED_E_CUDA;
  const int w = c.head_dim < 64 ? c.head_dim : 64, rows = c.page_size < kTile ? c.page_size : kTile;
  const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size, (cuuint64_t)c.n_kv_heads, (cuuint64_t)c.n_pages};
  // (the stride of a dimension of one entry is never used; the encoder wants a valid one)
  const auto bytes = [&](int i, int n) { return (cuuint64_t)(n == 1 && stride[i] == 0 ? c.head_dim : stride[i]) * 2; };
  const cuuint64_t strides[3] = {bytes(1, c.page_size), bytes(2, c.n_kv_heads), bytes(0, c.n_pages)};
  const cuuint32_t box[4] = {(cuuint32_t)w, (cuuint32_t)rows, 1, 1}, es[4] = {1, 1, 1, 1};
  const CUresult r = fn(m, type == ATSPEED_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
                        const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        w * 2 == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ATSPEED_OK : ATSPEED_E_ARG;
}

template <int HD>
atspeed_status launch(const CUtensorMap& mk, const CUtensorMap& mv, const TreeAttnArgs& a, int grid, cudaStream_t st) {
  static std::atomic<unsigned long long> done{0};
  if (smem_attr_once(done, tree_attention_kernel<HD>, Cfg<HD>::SMEM) != cudaSuccess) return ATSPEED_E_CUDA;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeCooperative;
  at[0].val.cooperative = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Cfg<HD>::SMEM;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, tree_attention_kernel<HD>, mk, mv, a) == cudaSuccess ? ATSPEED_OK : ATSPEED_E_CUDA;
}

int sm_count() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  return gemm_grid_size(dev);
}

constexpr size_t kCounterBytes = 2 * kMaxCtas * sizeof(int);

}  // namespace

unsigned int* tree_attn_err_word() {
  void* p = nullptr;
  return cudaGetSymbolAddress(&p, g_tree_attn_err) == cudaSuccess ? static_cast<unsigned int*>(p) : nullptr;
}

}  // namespace atspeed

using namespace atspeed;

extern "C" {

size_t atspeed_op_tree_attention_workspace(void) {
  const int n = sm_count();
  return kCounterBytes + (size_t)2 * (n < kMaxCtas ? n : kMaxCtas) * Cfg<128>::PART;
}

atspeed_status atspeed_op_tree_attention(atspeed_stream stream, const atspeed_kv_pages* cache, const void* d_q,
                                         int64_t q_stride, int n_heads, int n_req, int T, const int32_t* d_cu_q,
                                         const int32_t* d_ctx_len, const int32_t* d_block_table, int table_width,
                                         const uint32_t* d_mask, int mask_words, float scale, void* d_out, int64_t out_stride,
                                         float* d_lse, void* d_ws) {
  const atspeed_status ps_ok = check_pages(cache);
  if (ps_ok != ATSPEED_OK) return ps_ok;
  const atspeed_kv_pages& c = *cache;
  if (!d_q || !d_out || !d_cu_q || !d_ctx_len || !d_block_table || !d_ws || n_heads <= 0 || n_req <= 0 || T <= 0 ||
      table_width <= 0 || (d_mask && mask_words <= 0) || !(scale > 0.f) || !std::isfinite(scale))
    return ATSPEED_E_ARG;
  const int hd = c.head_dim, ps = c.page_size;
  if ((hd != 32 && hd != 64 && hd != 128) || (ps != 16 && ps != 32 && ps != 64 && ps != 128 && ps != 256) ||
      n_heads % c.n_kv_heads || n_heads / c.n_kv_heads > 128 || n_req > kMaxRequests || (long long)T * n_heads > 0x3fffffffLL)
    return ATSPEED_E_SHAPE;
  if (q_stride < (int64_t)n_heads * hd || out_stride < (int64_t)n_heads * hd || q_stride % 8 || out_stride % 8 ||
      !aligned16(d_q) || !aligned16(d_out) || (reinterpret_cast<uintptr_t>(d_ws) & 255))
    return ATSPEED_E_ARG;
  CUtensorMap mk, mv;
  atspeed_status st = page_map(&mk, c.d_k, c.k_type, c, c.k_stride);
  if (st == ATSPEED_OK) st = page_map(&mv, c.d_v, c.v_type, c, c.v_stride);
  if (st != ATSPEED_OK) return st;
  TreeAttnArgs a = {};
  a.q = static_cast<const uint16_t*>(d_q), a.v = static_cast<const uint16_t*>(c.d_v);
  for (int i = 0; i < 3; ++i) a.vs[i] = c.v_stride[i];
  a.q_stride = q_stride, a.out_stride = out_stride;
  a.H = n_heads, a.Hkv = c.n_kv_heads, a.G = n_heads / c.n_kv_heads, a.n = n_req, a.T = T, a.page = ps;
  a.width = table_width, a.words = mask_words, a.cu_q = d_cu_q, a.ctx = d_ctx_len, a.table = d_block_table, a.mask = d_mask;
  const long long cap = (long long)table_width * ps;
  a.cap = (int)(cap < (1LL << 30) ? cap : 1LL << 30);
  a.c = scale * 1.4426950408889634f;
  a.out = static_cast<uint16_t*>(d_out), a.lse = d_lse;
  a.k_f16 = c.k_type == ATSPEED_F16, a.v_f16 = c.v_type == ATSPEED_F16;
  a.arrived = static_cast<int*>(d_ws), a.done = a.arrived + kMaxCtas;
  a.parts = static_cast<unsigned char*>(d_ws) + kCounterBytes;
  a.err = tree_attn_err_word();
  const int grid = sm_count();
  if (!a.err || grid <= 0 || grid > kMaxCtas) return ATSPEED_E_CUDA;
  if (hd == 32) return launch<32>(mk, mv, a, grid, (cudaStream_t)stream);
  if (hd == 64) return launch<64>(mk, mv, a, grid, (cudaStream_t)stream);
  return launch<128>(mk, mv, a, grid, (cudaStream_t)stream);
}

}  // extern "C"
