// Attention of new tokens (trees, chains) over a batch's paged caches (atspeed_op_tree_attention), on the tensor cores.
//   o = sum_j w_j v_j / sum_j w_j, w_j = exp(scale q.k_j), over the positions j < ctx and those of the token's ancestors
//
// The rows of a (request, key head) are its new tokens times the G query heads that share the key head: they read the same
// K and V, so a block of up to 256 rows (two tiles of 128, or of the largest multiple of G below) reads each K / V tile of
// 128 keys once.  A tile is two products on tcgen05 with M =
// 128 rows: S = Q K^T (both K-major in shared memory) into TMEM, and O += P V with P (16 bits) as TMEM operand over S's
// columns and V in place, MN-major.  One thread a row runs the softmax from TMEM: no shuffles, no shared memory; O is scaled
// only where the running maximum rises by more than 2^8 (all weights are relative to the maximum in use, or to 2^-7 of it where
// they are rounded to fp16, so the quotient is the same).
//
// Two streams of (S, P, O) share the tensor core, each with a warp that issues its products and a warpgroup that runs its
// softmax.  Blocks of more than 128 rows: a stream is 128 of the rows, each sees every tile.  Fewer: both hold the same rows
// and take alternate tiles; they are joined at the end.  (Padding a single token's G rows to 128 costs tensor time that the
// tile's 64 KB of K and V, 2800 clocks of an SM's share of the HBM, leave free.)
//
// P goes out in two halves of 64 keys, so that the first half's product runs under the second half's exponentials.  (Tiles of
// 64 keys with two S a stream, so that a softmax never waits for its S, lose more than they gain: a product of N = 64 takes the
// tensor core the 64 clocks of one of N = 128.  Two threads a row made the softmax no faster.)
//
// Work is the concatenation of all blocks' tiles, each block's with a cost in front, cut into one equal range a CTA (every CTA
// finds its own range from the lengths; an end next to a block's border is moved there).  A block that an end cuts is summed
// from partial results in device memory, each of its CTAs taking a share of the rows, in range order.  Waits for partial
// results come after all own results are out and the grid is launched cooperatively, so that they end; they are bounded all
// the same.
//
// Bound and measured: few rows over long caches by HBM (61 single tokens over 500 to 16 000 keys, 32 heads on 8 of 128: 188 us,
// 6.2 TB/s); many rows by the streams' chain S, maximum, exponentials (1000 of 2900 clocks a tile), P, O, not by the tensor
// pipe (29 to 43% busy): 16 trees of 240 tokens 82 us, 515 TFLOP/s; a prompt of 2 x 4001 tokens, heads of 64, 315 us, 772 TFLOP/s.
// A single token over 512 keys takes 13.7 us, all latency.
//
// Roles (384 threads): warp 0 copies (TMA), warps 1 and 2 issue the products of a stream each, warp 3 loads Q, warps 4-7 and
// 8-11 run the streams' softmax.  A stream's warps keep their place in the walk over the blocks in shared memory: beside a
// row of S it does not fit the registers, and spilled it cost 20 to 75% of the time where the HBM is the bound (8 to 12 bytes
// of a thread's still are spilled).
#include <cuda.h>
#include <cudaTypedefs.h>

#include <cmath>

#include "common.cuh"
#include "gemm.cuh"
#include "step_ops.cuh"

namespace atspeed {
namespace {

__device__ unsigned int g_tree_attn_err;

constexpr int kThreads = 384, kStreamThreads = 256;
constexpr int kTile = 128;       // keys of a tile
constexpr int kBlock = 256;      // rows of a block, at most
constexpr int kRoleRegs = 88, kStreamRegs = 208;
static_assert(128 * kRoleRegs + kStreamThreads * kStreamRegs <= kThreads * 168, "registers at launch");
constexpr float kSlack = 8.f;    // rise of the running maximum (log2) below which O keeps its scale
// Where V and so P are fp16, weights are relative to 2^-7 of the maximum in use: fp16 ends at 2^-24 and the largest P would be
// 2^kSlack of its 2^16, so that weights below 2^-25 of a large one would be 0 in P V, however many they are (20 000 keys 17.4 nats
// below one whose V is 0: 100% off; with this below 1%, down to the 2^-32 of the maximum where a weight has no bits).
constexpr float kRaise = 7.f;
static_assert(kSlack + kRaise <= 15.f, "P in fp16");
constexpr int kWalkBytes = 80;   // of a warp's place in the walk
constexpr int kLeastUnits = 2;   // of a CTA's range (1: 2 to 14% slower over ten small calls, 3: 10 to 30% on most)
constexpr int kMaxCtas = 256;    // of a grid: counters in the workspace, and a share's weights in shared memory (below)

template <int HD>
struct Cfg {
  static constexpr int SW = HD >= 64 ? 128 : 64;       // bytes of a panel's row, and its swizzle
  static constexpr int PANELS = HD * 2 / SW;
  static constexpr int PANEL = kTile * SW, Q_PANEL = 128 * SW;
  static constexpr int TILE = PANELS * PANEL, Q_TILE = PANELS * Q_PANEL;   // K or V tile; 128 rows of Q
  static constexpr int STAGES = HD == 128 ? 5 : 8;
  static constexpr int Q_OFF = STAGES * TILE;
  static constexpr int X_OFF = Q_OFF + 2 * Q_TILE;       // (m, l) of both streams' rows
  static constexpr int X_BYTES = kStreamThreads * 8;     // .. and, when they are done, the weights of a share of a cut block
  // (a share of 1 / parts of a block's rows, rounded up, by parts: at most rows + parts - 1 weights)
  static_assert((kBlock + kMaxCtas - 1) * (int)sizeof(float) <= X_BYTES, "weights of a share");
  static constexpr int BAR_OFF = X_OFF + X_BYTES;
  static constexpr int WALK_OFF = BAR_OFF + 256, START_OFF = WALK_OFF + 8 * kWalkBytes;
  static constexpr int SMEM = START_OFF + 64;
  static constexpr int S_COL = 128, O_COL = 256;       // TMEM columns: S / P of stream s at s * 128, O at 256 + s * HD
  static constexpr int O_STEP = HD;
  static constexpr size_t PART = (size_t)kBlock * (HD + 2) * 4;   // bytes of a partial result: O [256][HD], (m, l) [256]
};
static_assert(Cfg<128>::SMEM <= 232448 && Cfg<64>::SMEM <= 232448, "shared memory of a CTA");

struct TreeAttnArgs {
  const uint16_t* v;
  long long vs[3], out_stride;
  int H, Hkv, G, n, T, page, page_log, n_pages, width, words;
  int cap;                                        // positions that a table row covers
  int rt, block_tokens;                           // rows of a stream's tile: the multiple of G up to 128; tokens of a block
  const int *cu_q, *ctx, *table;
  const uint32_t* mask;
  float c;                                        // scale * log2(e)
  uint16_t* out;
  float* lse;
  bool k_f16, v_f16, out32;                       // out32: rows of the output begin at multiples of 32 bytes
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
  r.blocks = r.ctx < 0 ? 0 : (r.q + a.block_tokens - 1) / a.block_tokens;
  return r;
}
__device__ __forceinline__ int block_keys(const TreeAttnArgs& a, const Request& r, int blk) {
  const int last = a.mask ? r.q : min(r.q, (blk + 1) * a.block_tokens);
  return (int)min((long long)r.ctx + last, (long long)a.cap);
}
__device__ __forceinline__ int tiles_of(int keys) { return (keys + kTile - 1) / kTile; }
__device__ __forceinline__ int block_rows(const TreeAttnArgs& a, const Request& r, int blk) {
  return min(2 * a.rt, r.rows - blk * 2 * a.rt);
}
// What a block costs beside its tiles (its Q, its pipeline's start, its masks and its result), in tiles, so that ranges of equal
// units take equal times.  Measured at heads of 128, against no cost at all: 61 single tokens 208 -> 188 us with 1 (a CTA has
// up to three blocks, another one long one); 16 trees of 240 tokens 107 -> 99 us with 2 to 6; a causal prompt of 4001 tokens
// loses instead, 390 -> 403 us (its blocks are all of one kind and long).  Since ends move to blocks' borders (below) trees of
// 240 tokens are the same either way; 40 of 60 tokens, 32 heads on 8 of 128 / 64 / 32, took 84.6 / 68.3 / 60 us with no cost and
// 82.6 / 64.2 / 58 like this, the 61 single tokens 215 / 166 / 139 and 212 / 160 / 136 (cold L2).
__device__ __forceinline__ int block_cost(const TreeAttnArgs& a, const Request& r, int blk) {
  return block_rows(a, r, blk) <= a.rt ? 1 : a.mask ? 4 : 0;
}
__device__ __forceinline__ int block_units(const TreeAttnArgs& a, const Request& r, int blk) {
  return block_cost(a, r, blk) + tiles_of(block_keys(a, r, blk));
}
__device__ __forceinline__ long long request_units(const TreeAttnArgs& a, const Request& r) {
  if (r.blocks == 0) return 0;
  long long u = block_units(a, r, r.blocks - 1);
  if (a.mask) u += (r.blocks - 1LL) * block_units(a, r, 0);
  else
    for (int i = 0; i < r.blocks - 1; ++i) u += block_units(a, r, i);
  return u * a.Hkv;
}

// x / d, of numbers that are small as a rule
__device__ __forceinline__ long long quotient(long long x, long long d) {
  return (unsigned long long)(x | d) >> 32 ? x / d : (long long)((unsigned)x / (unsigned)d);
}
// How far a range's end may be moved to a block's border, so that the block is not cut for it (a cut block of 256 rows costs each
// of its CTAs some 5 us: 132 KB out, a wait, its share back in); `most`: a sixth of the range.  Measured, heads of 128, against
// no move: 512 blocks of 16 trees 97 -> 82 us; heads of 64: a prompt 317 -> 309; looking for both of a range's ends costs a
// call of one token 1.2 us (13.4 -> 14.6).
__device__ __forceinline__ int block_slack(const TreeAttnArgs& a, int rows, int most) {
  return min(rows > a.rt ? 6 : 1, most);
}

struct Start {      // a CTA's range: where it begins
  long long u0, u1, units;
  int b, kh, blk, off, ctas;   // (off: units into the block)
  int most;                    // of block_slack
};

struct Walk {
  Request r;
  long long left;     // units of the range from this block on
  long long begin;    // the block's first unit
  int b, kh, blk;
  int tile0, tiles;   // this CTA's tiles of the block
  int all, keys;      // tiles and keys of the whole block
  int rows;           // rows of the block
  int cost, units;    // its cost, and the range's units in it
  __device__ __forceinline__ void start(const TreeAttnArgs& a, const Start& s) {
    left = s.u1 - s.u0, b = s.b, kh = s.kh, blk = s.blk, tiles = 0;
    if (left <= 0) return;
    r = request(a, b);
    begin = s.u0 - s.off;
    block(a, s.off);
    if (units == 0) next(a);
  }
  // A block's units are its cost's, which are no work, and its tiles' after them.
  __device__ __forceinline__ void block(const TreeAttnArgs& a, int off) {
    keys = block_keys(a, r, blk);
    all = tiles_of(keys);
    rows = block_rows(a, r, blk);
    cost = block_cost(a, r, blk);
    units = (int)min((long long)(cost + all - off), left);
    tile0 = max(0, off - cost);
    tiles = max(0, off + units - cost) - tile0;
  }
  __device__ bool more() const { return left > 0 && tiles > 0; }
  __device__ __forceinline__ void next(const TreeAttnArgs& a) {
    left -= units;
    begin += cost + all;
    if (left <= 0) return;
    if (++blk == r.blocks) {
      blk = 0;
      if (++kh == a.Hkv) {
        kh = 0;
        do r = request(a, ++b);
        while (r.blocks == 0 && b < a.n - 1);
      }
    }
    block(a, 0);
  }
  __device__ bool dual(const TreeAttnArgs& a) const { return rows > a.rt; }
};
static_assert(sizeof(Walk) <= kWalkBytes, "a warp's place in shared memory");

// ---------------------------------------------------------------------------------------------
// instructions
// ---------------------------------------------------------------------------------------------
// (by the thread with `lead`: issued by several lanes at once, a copy's operands are moved to uniform registers lane by lane)
__device__ __forceinline__ void tma_load_4d(uint32_t lead, uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z,
                                            int w) {
  asm volatile(
      "{\n .reg .pred e;\n setp.ne.b32 e, %7, 0;\n @e cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::"
      "complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n}" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar), "r"(lead)
      : "memory");
}
// One product of 16 along K, by the thread with `lead`.  Descriptors come as their low words (address, lead offset) and the
// high word that all operands of a kernel share.  A in shared memory, or in TMEM.
__device__ __forceinline__ void mma_ss(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t idesc,
                                       uint32_t add) {
  asm volatile(
      "{\n .reg .pred e, p;\n .reg .b64 da, db;\n setp.ne.b32 e, %6, 0;\n setp.ne.b32 p, %5, 0;\n"
      " mov.b64 da, {%1, %3};\n mov.b64 db, {%2, %3};\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n}" ::"r"(d),
      "r"(a), "r"(b), "r"(hi), "r"(idesc), "r"(add), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t idesc,
                                       uint32_t add) {
  asm volatile(
      "{\n .reg .pred e, p;\n .reg .b64 db;\n setp.ne.b32 e, %6, 0;\n setp.ne.b32 p, %5, 0;\n"
      " mov.b64 db, {%2, %3};\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n}" ::"r"(d),
      "r"(a), "r"(b), "r"(hi), "r"(idesc), "r"(add), "r"(lead)
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
// wait::ld with the registers it is about, so that nothing that uses them moves ahead of it
__device__ __forceinline__ void tmem_ld_wait128(uint32_t (&x)[128]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int j = 0; j < 128; j += 16)
    asm volatile(""
                 : "+r"(x[j]), "+r"(x[j + 1]), "+r"(x[j + 2]), "+r"(x[j + 3]), "+r"(x[j + 4]), "+r"(x[j + 5]), "+r"(x[j + 6]),
                   "+r"(x[j + 7]), "+r"(x[j + 8]), "+r"(x[j + 9]), "+r"(x[j + 10]), "+r"(x[j + 11]), "+r"(x[j + 12]),
                   "+r"(x[j + 13]), "+r"(x[j + 14]), "+r"(x[j + 15]));
}
__device__ __forceinline__ void tmem_ld_wait16(uint32_t (&x)[16], uint32_t (&y)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int j = 0; j < 16; j += 8)
    asm volatile(""
                 : "+r"(x[j]), "+r"(x[j + 1]), "+r"(x[j + 2]), "+r"(x[j + 3]), "+r"(x[j + 4]), "+r"(x[j + 5]), "+r"(x[j + 6]),
                   "+r"(x[j + 7]), "+r"(y[j]), "+r"(y[j + 1]), "+r"(y[j + 2]), "+r"(y[j + 3]), "+r"(y[j + 4]), "+r"(y[j + 5]),
                   "+r"(y[j + 6]), "+r"(y[j + 7]));
}
// 32 bytes, a whole sector, by one thread
__device__ __forceinline__ void st_global_32(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
               "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void hold64(uint32_t* x) {
#pragma unroll
  for (int j = 0; j < 64; j += 16)
    asm volatile(""
                 : "+r"(x[j]), "+r"(x[j + 1]), "+r"(x[j + 2]), "+r"(x[j + 3]), "+r"(x[j + 4]), "+r"(x[j + 5]), "+r"(x[j + 6]),
                   "+r"(x[j + 7]), "+r"(x[j + 8]), "+r"(x[j + 9]), "+r"(x[j + 10]), "+r"(x[j + 11]), "+r"(x[j + 12]),
                   "+r"(x[j + 13]), "+r"(x[j + 14]), "+r"(x[j + 15]));
}
// The instruction, good to 2^-22: below what P's 16 bits keep, and in the joins below the roundings of P that they sum.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two values at once: x * m + a, and x + y (in 32 bits each).
__device__ __forceinline__ float2 fma2(float2 x, float2 m, float2 a) {
  float2 y;
  asm("{\n .reg .b64 r, s, t;\n mov.b64 r, {%2, %3};\n mov.b64 s, {%4, %5};\n mov.b64 t, {%6, %7};\n"
      " fma.rn.f32x2 r, r, s, t;\n mov.b64 {%0, %1}, r;\n}"
      : "=f"(y.x), "=f"(y.y)
      : "f"(x.x), "f"(x.y), "f"(m.x), "f"(m.y), "f"(a.x), "f"(a.y));
  return y;
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  float2 z;
  asm("{\n .reg .b64 r, s;\n mov.b64 r, {%2, %3};\n mov.b64 s, {%4, %5};\n add.rn.f32x2 r, r, s;\n mov.b64 {%0, %1}, r;\n}"
      : "=f"(z.x), "=f"(z.y)
      : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
  return z;
}
__device__ __forceinline__ void named_bar_arrive(int id, int nthreads) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(nthreads) : "memory");
}
__device__ __forceinline__ int warp_uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// Shared-memory descriptors (fields: common.cuh, smem_desc_sw128): the low word holds the address and `lead`, the bytes
// between panels of an MN-major operand wider than one; the high word the bytes between groups of eight rows of a panel,
// the version and the swizzle (2: 128 bytes, 4: 64).
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lead) {
  return ((addr >> 4) & 0x3FFFu) | ((lead >> 4) & 0x3FFFu) << 16;
}
template <int SW>
constexpr uint32_t kDescHi = ((8u * SW) >> 4) | 1u << 14 | (SW == 128 ? 2u : 4u) << 29;
// Instruction descriptor (fields: idesc_bf16_f32); bit 16: B is MN-major
__device__ __forceinline__ uint32_t instr_desc(int n, bool f16, bool b_mn) {
  const uint32_t t = f16 ? 0u : 1u;
  return (1u << 4) | (t << 7) | (t << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}

// Place of a K or V tile in the order of the copies, of a range of n tiles: K runs ahead of V by the S that are under way (one
// tile where both streams see every tile, two where they alternate), then V and K take turns: K0 .. K(L-1), V0, K(L), V1, ..
__device__ __forceinline__ int k_lead(bool dual) { return dual ? 1 : 2; }
__device__ __forceinline__ int seq_k(int lead, int i) { return i < lead ? i : 2 * i - lead + 1; }
__device__ __forceinline__ int seq_v(int lead, int i, int n) { return min(lead, n) + i + min(i, max(0, n - lead)); }

__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// The 32 NW keys from `key` on that token i of request r sees, lowest bit first.
template <int NW>
__device__ __forceinline__ void seen_keys(const TreeAttnArgs& a, const Request& r, int i, int key, uint32_t (&x)[NW]) {
  const int j0 = key - r.ctx;   // first of them among the new tokens; below 0 there are cached positions
  if (a.mask) {
    const uint32_t* row = a.mask + (long long)(r.t0 + i) * a.words;
    const int w = j0 >> 5, sh = j0 & 31;   // (arithmetic: j0 may be negative)
    uint32_t m[NW + 1];
#pragma unroll
    for (int k = 0; k <= NW; ++k) m[k] = w + k >= 0 && w + k < a.words ? __ldg(row + w + k) : 0u;
#pragma unroll
    for (int k = 0; k < NW; ++k) x[k] = __funnelshift_r(m[k], m[k + 1], sh) & low_bits(r.q - j0 - 32 * k);
  } else {
#pragma unroll
    for (int k = 0; k < NW; ++k) x[k] = low_bits(i + 1 - j0 - 32 * k);
  }
#pragma unroll
  for (int k = 0; k < NW; ++k) x[k] = (x[k] | low_bits(-j0 - 32 * k)) & low_bits(a.cap - key - 32 * k);
}

// Of a V tile's keys those from `first` on: NaN and infinities become 0, in every key; *odd is set if one was found before
// key `last`.  By 128 threads.  (Two 16-bit values are tested at once: with its sign off, a value that is not finite plus
// `step` reaches the sign's place.)
template <int HD>
__device__ __forceinline__ void clean_v(uint8_t* v0, int r, int first, int last, bool f16, volatile int* odd) {
  using C = Cfg<HD>;
  constexpr int RC = C::SW / 16;   // 16-byte chunks of a panel's row
  const uint32_t step = f16 ? 0x04000400u : 0x00800080u;
  const auto beyond = [&](uint32_t two) { return (two & 0x7fff7fffu) + step & 0x80008000u; };
  uint4* chunk = reinterpret_cast<uint4*>(v0) + r % RC;
  uint32_t any = 0;
#pragma unroll 4
  for (int row = first + r / RC; row < kTile; row += 128 / RC)
#pragma unroll
    for (int panel = 0; panel < C::PANELS; ++panel) {
      const uint4 v = chunk[(panel * C::PANEL + row * C::SW) / 16];
      any |= beyond(v.x) | beyond(v.y) | beyond(v.z) | beyond(v.w);
    }
  if (!any) return;
#pragma unroll 1
  for (int panel = 0; panel < C::PANELS; ++panel)
#pragma unroll 1
    for (int row = first + r / RC; row < kTile; row += 128 / RC) {
      uint16_t* v = reinterpret_cast<uint16_t*>(chunk + (panel * C::PANEL + row * C::SW) / 16);
#pragma unroll 1
      for (int j = 0; j < 8; ++j) {
        if (!beyond(v[j])) continue;
        if (row < last) {
          *odd = 1;
          __threadfence_block();
        }
        v[j] = 0;
      }
    }
  fence_proxy_async_shared();
}

// The NaN and infinities of V that a row sees among keys [p0, p1) and that were 0 in its tiles, added to columns [c0, c1) of
// its result in device memory (the call's output, or a partial result in 32 bits).
template <int HD>
__device__ __noinline__ void add_odd_v(const TreeAttnArgs& a, int b, int kh, int tok, int p0, int p1, int c0, int c1, uint16_t* out,
                                       float* part) {
  const Request r = request(a, b);
  for (int p = p0; p < p1; ++p) {
    uint32_t see[1];
    seen_keys(a, r, tok, p, see);
    if (!(see[0] & 1)) continue;
    const int id = a.table[(long long)b * a.width + (p >> a.page_log)];
    if (id < 0 || id >= a.n_pages) continue;
    const uint16_t* v = a.v + id * a.vs[0] + (p & (a.page - 1)) * a.vs[1] + kh * a.vs[2];
    for (int c = c0; c < c1; ++c) {
      const float x = unpack2(v[c], a.v_f16).x;
      if (isfinite(x)) continue;
      if (part) part[c] += x;
      else out[c] = (uint16_t)pack2(unpack2(out[c], a.k_f16).x + x, 0.f, a.k_f16);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// a partial result's place, and the block's CTAs
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ int cta_of(long long u, const Start& s) { return (int)quotient((u + 1) * s.ctas - 1, s.units); }

template <int HD>
__device__ __forceinline__ float* part_of(const TreeAttnArgs& a, int cta, int slot) {
  return reinterpret_cast<float*>(a.parts + (size_t)(2 * cta + slot) * Cfg<HD>::PART);
}

// Rows [row0, row0 + n) of a cut block, four columns a thread at a time: U of them side by side and the parts in steps of P, so
// that U P loads are under way; the parts are added in their order either way.
template <int HD, int U, int P, typename Place>
__device__ __forceinline__ void sum_parts(const TreeAttnArgs& a, int first, int parts, int n, int row0, int tid, const float* w,
                                          const Place& place) {
  constexpr int V4 = HD / 4;
  for (int i0 = tid; i0 < n * V4; i0 += U * kStreamThreads) {
    float4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u) o[u] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int q = 0; q < parts; q += P) {
      float4 y[P][U];
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (q + p < parts && i0 + u * kStreamThreads < n * V4)
            y[p][u] = __ldcg(reinterpret_cast<const float4*>(part_of<HD>(a, first + q + p, q + p == 0) + row0 * HD) + i0 + u * kStreamThreads);
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (q + p >= parts || i0 + u * kStreamThreads >= n * V4) continue;
          const float f = w[(i0 + u * kStreamThreads) / V4 * parts + q + p];
          o[u].x += f * y[p][u].x, o[u].y += f * y[p][u].y, o[u].z += f * y[p][u].z, o[u].w += f * y[p][u].w;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kStreamThreads;
      if (i >= n * V4) continue;
      int t, h;
      place(row0 + i / V4, t, h);
      *reinterpret_cast<uint2*>(a.out + (long long)t * a.out_stride + (long long)h * HD + i % V4 * 4) =
          make_uint2(pack2(o[u].x, o[u].y, a.k_f16), pack2(o[u].z, o[u].w, a.k_f16));
    }
  }
}

// A CTA's share of a cut block's rows: the sum of the partial results in their order, by both streams' threads.  First every
// part's weight in every row of the share, into shared memory (at most 256 + parts - 1 of them, however many of each);
// then four columns a thread, several loads under way.  (8 query heads over 16 000 keys of one key head, 63 parts: 61 us with a
// thread a row and two loads under way and ranges of one unit, 21 like this.)
template <int HD>
__device__ __forceinline__ void merge_share(const TreeAttnArgs& a, const Request& r, int kh, int blk, int first, int parts,
                                            int share, int tid, float* w) {
  constexpr int V4 = HD / 4;
  const int rows = min(2 * a.rt, r.rows - blk * 2 * a.rt);
  const int row0 = rows * share / parts, n = rows * (share + 1) / parts - row0;
  const auto place = [&](int row, int& t, int& h) {
    const int rg = blk * 2 * a.rt + row;
    t = r.t0 + rg / a.G, h = kh * a.G + rg % a.G;
  };
  // Weights: a thread a row, or, of many parts (and so few rows), a warp a row.
  const bool wide = parts >= 16;
  const int lane = tid & 31, p0 = wide ? lane : 0, step = wide ? 32 : 1;
  for (int i = wide ? tid >> 5 : tid; i < n; i += wide ? kStreamThreads / 32 : kStreamThreads) {
    const auto ml = [&](int p) {
      return __ldcg(reinterpret_cast<const float2*>(part_of<HD>(a, first + p, p == 0) + kBlock * HD) + row0 + i);
    };
    float m = -INFINITY, l = 0.f;
#pragma unroll 4
    for (int p = p0; p < parts; p += step) m = fmaxf(m, ml(p).x);
    if (wide)
      for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll 4
    for (int p = p0; p < parts; p += step) {
      // (a part that saw none of the row's keys has l = 0 and no scale; a NaN in l stays one)
      const float2 x = ml(p);
      const float f = x.x == -INFINITY ? x.y : exp2_fast(x.x - m);
      l += x.x == -INFINITY ? x.y : f * x.y;
      w[i * parts + p] = f;
    }
    if (wide)
      for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    for (int p = p0; p < parts; p += step) w[i * parts + p] *= inv;
    if (a.lse && p0 == 0) {
      int t, h;
      place(row0 + i, t, h);
      a.lse[(long long)t * a.H + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
    }
  }
  named_bar_sync(1, kStreamThreads);
  if (n * V4 <= kStreamThreads) sum_parts<HD, 1, 8>(a, first, parts, n, row0, tid, w, place);
  else sum_parts<HD, 4, 2>(a, first, parts, n, row0, tid, w, place);
}

__device__ __forceinline__ bool wait_count(const int* p, int want, unsigned int* err) {
  const unsigned long long t0 = globaltimer_ns();
  for (unsigned it = 1;; ++it) {
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    if (v >= want) return true;
    __nanosleep(100);   // (a CTA that is early must not take the memory system's time from those that are not)
    if ((it & 255u) == 0u && globaltimer_ns() - t0 > kWaitBudgetNs) {
      set_error(err, ATSPEED_DEV_ERR_TIMEOUT);
      return false;
    }
  }
}

// Whether a phase of a barrier of this CTA is complete.
__device__ __forceinline__ bool bar_done(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok)
               : "r"(smem_u32(bar)), "r"(parity)
               : "memory");
  return ok != 0;
}
// A wait of a whole warp, which goes on together; after the first that gave up the rest are not waited for (the loops run
// to their ends without the work, so that every barrier meets its threads).
__device__ __forceinline__ bool warp_wait(bool ok, uint64_t* bar, uint32_t parity, unsigned int* err) {
  if (__builtin_expect(__all_sync(0xffffffffu, bar_done(bar, parity)), 1) || !ok) return ok;
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, err));
}

template <int HD, bool KF16, bool VF16>
__global__ void __launch_bounds__(kThreads, 1)
    tree_attention_kernel(const __grid_constant__ CUtensorMap tmq, const __grid_constant__ CUtensorMap tmk,
                          const __grid_constant__ CUtensorMap tmv, const __grid_constant__ TreeAttnArgs a) {
  using C = Cfg<HD>;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::BAR_OFF);
  uint64_t* empty = full + C::STAGES;
  uint64_t* s_full = empty + C::STAGES;   // [2] S of a stream is in TMEM (and the P V before it complete)
  uint64_t* p_ready = s_full + 2;         // [2][2] the halves of its P are
  uint64_t* q_full = p_ready + 4;
  uint64_t* q_free = q_full + 1;
  uint64_t* o_done = q_free + 1;          // the block's products are complete
  uint64_t* o_free = o_done + 1;          // its O is read
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_free + 1);
  volatile int* odd_v = reinterpret_cast<int*>(tmem_slot + 1);   // a NaN or infinity was found in a new token's V
  Start* start = reinterpret_cast<Start*>(smem + C::START_OFF);
  const int tid = threadIdx.x, warp = warp_uniform(tid >> 5), lane = tid & 31;
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
    sums[kThreads / 32 + tid] = sum - own, sums[kThreads / 32 + kThreads + tid] = own;
    if (warp == 3) tmem_alloc(tmem_slot, 512);
    if (tid == 0) {
      for (int i = 0; i < C::STAGES; ++i) mbar_init(full + i, 1), mbar_init(empty + i, 2);
      for (int i = 0; i < 2; ++i) mbar_init(s_full + i, 1);
      for (int i = 0; i < 4; ++i) mbar_init(p_ready + i, 4);
      mbar_init(q_full, 1);
      mbar_init(q_free, 2);
      mbar_init(o_done, 2);
      mbar_init(o_free, kStreamThreads / 32);
      fence_mbar_init();
      *odd_v = 0;
      start->u0 = start->u1 = 0;
    }
    if (tid == 32) tma_prefetch_desc(&tmq), tma_prefetch_desc(&tmk), tma_prefetch_desc(&tmv);
    __syncthreads();
    // (another thread looks for the range's end among the requests of this one)
    const int other = tid < kThreads / 2 ? tid + kThreads / 2 : tid - kThreads / 2;
    long long total = 0, before = sum - own, before1 = sums[kThreads / 32 + other];
    const long long own1 = sums[kThreads / 32 + kThreads + other];
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) before += sums[w];
      if (w < other >> 5) before1 += sums[w];
      total += sums[w];
    }
    const int ctas = (int)min((long long)gridDim.x, (total + kLeastUnits - 1) / kLeastUnits), cta = blockIdx.x;
    if (cta < ctas) {
      const long long u0 = quotient(cta * total, ctas), u1 = quotient((cta + 1LL) * total, ctas);
      const int most = (int)min(quotient(total, ctas * 6), 1LL << 20);
      // The block that holds a unit, and how far into it the border at that unit is, moved where that saves a cut.
      const auto find = [&](long long off, int first, int& b, int& kh, int& blk) {
        Request r;
        for (b = first;; ++b) {
          r = request(a, b);
          const long long x = request_units(a, r);
          if (off < x) {
            const long long head = quotient(x, a.Hkv);
            kh = (int)quotient(off, head), off -= kh * head, blk = 0;
            break;
          }
          off -= x;
        }
        int units;
        for (; off >= (units = block_units(a, r, blk)); ++blk) off -= units;
        const int slack = block_slack(a, block_rows(a, r, blk), most);
        return off <= slack ? make_int2((int)off, 0) : make_int2((int)off, units - off <= slack ? units : (int)off);
      };
      if (u0 >= before && u0 < before + own) {
        const int2 x = find(u0 - before, b0, start->b, start->kh, start->blk);
        start->off = x.y;
        start->u0 = u0 - x.x + x.y, start->units = total, start->ctas = ctas, start->most = most;
      }
      if (u1 == total ? tid == 0 : u1 >= before1 && u1 < before1 + own1) {
        int b, kh, blk;
        const int2 x = u1 == total ? make_int2(0, 0) : find(u1 - before1, min(a.n, other * per), b, kh, blk);
        start->u1 = u1 - x.x + x.y;
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
  const uint32_t tmem = warp_uniform(*tmem_slot);
  const Start st = *start;
  bool ok = true;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRoleRegs));
    if (warp == 0) {
      // ---- copies ----
      // A tile is copied page by page (or half a page of 256), a panel of 64 dimensions at a time.  The page numbers of 32
      // boxes are read at once, one a lane, the next 32 ahead of time.
      const uint32_t lead = elect_one(), ring = smem_u32(smem), bars = smem_u32(full);
      const int box_log = min(a.page_log, 7), n_box = kTile >> box_log;
      unsigned seq = 0;
      struct Pages {
        int now, next, base;   // of the 32 boxes from `base` on, and of the 32 after
      };
      Walk w;
      for (w.start(a, st); w.more(); w.next(a)) {
        const int n = warp_uniform(w.tiles), ahead = k_lead(warp_uniform(w.dual(a)));
        const int tile0 = warp_uniform(w.tile0), keys = warp_uniform(w.keys), kh = warp_uniform(w.kh);
        const int* table = a.table + (long long)w.b * a.width;
        const auto read = [&](int box) {   // this lane's of the 32 boxes from `box` on
          const int key = (box + lane) << box_log;
          return key < keys ? __ldg(table + (key >> a.page_log)) : 0;
        };
        const auto copy = [&](const CUtensorMap* map, int i, Pages& p) {
          const unsigned slot = seq % C::STAGES;
          const int key0 = (tile0 + i) * kTile, box0 = key0 >> box_log;
          const int boxes = min(n_box, (keys - key0 + (1 << box_log) - 1) >> box_log);
          if (box0 - p.base >= 32) p.now = p.next, p.base += 32, p.next = read(p.base + 32);
          ok = warp_wait(ok, empty + slot, (seq / C::STAGES & 1) ^ 1, err);
          ++seq;
          if (!ok) return;
          mbar_expect_tx_lead(lead, full + slot, (boxes << box_log) * HD * 2);
#pragma unroll 1
          for (int b = 0; b < boxes; ++b) {
            const int id = __shfl_sync(0xffffffffu, p.now, box0 + b - p.base);
#pragma unroll
            for (int panel = 0; panel < C::PANELS; ++panel)
              tma_load_4d(lead, ring + slot * C::TILE + panel * C::PANEL + (b << box_log) * C::SW, map, bars + slot * 8,
                          panel * (C::SW / 2), (key0 + (b << box_log)) & (a.page - 1), kh, id);
          }
        };
        Pages pk, pv;
        pk.base = pv.base = tile0 * n_box;
        pk.now = pv.now = read(pk.base);
        pk.next = pv.next = read(pk.base + 32);
#pragma unroll 1
        for (int i = -ahead; i < n; ++i) {   // V of tile i, K of tile i + ahead
          if (i >= 0) copy(&tmv, i, pv);
          if (i + ahead < n) copy(&tmk, i + ahead, pk);
        }
      }
    } else if (warp < 3) {
      // ---- products of a stream ----
      // (all that the products' operands are made of is the same in every lane, and said to be so: an operand that may
      // differ is moved to a uniform register anew for each product)
      const uint32_t lead = elect_one();
      const int s = warp - 1;
      const uint32_t id_s = instr_desc(kTile, KF16, false), id_o = instr_desc(HD, VF16, true), hi = kDescHi<C::SW>;
      const uint32_t ring = desc_lo(smem_u32(smem), C::PANEL), qs = desc_lo(smem_u32(smem + C::Q_OFF), C::Q_PANEL);
      const uint32_t t_s = tmem + s * C::S_COL, t_o = tmem + C::O_COL + s * C::O_STEP;
      unsigned seq0 = 0, item = 0, turn = 0, pos = 0;   // turn: tiles this stream has been through; pos: places
      // Every place of the ring up to `seq` is gone through in order.  Of the other stream's tiles that is all: their copy is
      // waited for and the place given back.  (A wait tells a phase from the next one only, by its parity: a place that is
      // filled again before this stream has seen it would be taken for the wrong copy.)
      const auto pass = [&](unsigned seq) {
        for (; pos < seq; ++pos) {
          ok = warp_wait(ok, full + pos % C::STAGES, pos / C::STAGES & 1, err);
          if (lane == 0 && ok) mbar_arrive(empty + pos % C::STAGES);
        }
      };
      Walk w;
      for (w.start(a, st); w.more(); w.next(a), ++item) {
        const bool dual = warp_uniform(w.dual(a));
        const int n = warp_uniform(w.tiles), tiles = dual ? n : (n - s + 1) / 2, ahead = k_lead(dual);
        const uint32_t qd = qs + (dual ? s * (C::Q_TILE >> 4) : 0);
        const auto copied = [&](unsigned seq) {
          if (pos > seq) return;
          pass(seq);
          ok = warp_wait(ok, full + seq % C::STAGES, seq / C::STAGES & 1, err);
          pos = seq + 1;
        };
        // The same as far as it takes no waiting.
        const auto copied_by_now = [&](unsigned seq) {
          for (; pos <= seq; ++pos) {
            if (!__all_sync(0xffffffffu, bar_done(full + pos % C::STAGES, pos / C::STAGES & 1))) return;
            if (pos < seq && lane == 0) mbar_arrive(empty + pos % C::STAGES);
          }
        };
        // (a stream without tiles waits too: no stream may be a block ahead on these barriers)
        ok = warp_wait(ok, q_full, item & 1, err);
        if (tiles == 0 && ok) tc_commit_lead(lead, q_free);
        // S of the stream's first tile, then P V of tile k and S of tile k + 1 in turn
#pragma unroll 1
        for (int k = -1; k < tiles; ++k) {
          const unsigned v_seq = seq0 + seq_v(ahead, dual ? k : 2 * k + s, n), v_slot = v_seq % C::STAGES;
          const unsigned k_seq = seq0 + seq_k(ahead, dual ? k + 1 : 2 * k + 2 + s), k_slot = k_seq % C::STAGES;
          if (k >= 0) {
            if (k == 0) ok = warp_wait(ok, o_free, (item & 1) ^ 1, err);
            copied(v_seq);
            if (k + 1 < tiles && ok) copied_by_now(k_seq);
            const uint32_t vd = ring + v_slot * (C::TILE >> 4);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              ok = warp_wait(ok, p_ready + 2 * s + h, (turn + k) & 1, err);
              if (!ok) continue;
              tc_fence_after();
#pragma unroll
              for (int j = 4 * h; j < 4 * h + 4; ++j)
                mma_ts(lead, t_o, t_s + j * 8, vd + (j * 16 * C::SW >> 4), hi, id_o, k > 0 || j > 0);
            }
          }
          if (k + 1 < tiles) {
            copied(k_seq);
            if (ok) {
              tc_fence_after();
              const uint32_t kd = ring + k_slot * (C::TILE >> 4);
#pragma unroll
              for (int j = 0; j < HD / 16; ++j) {
                const uint32_t step = ((j * 32 / C::SW) * C::PANEL + j * 32 % C::SW) >> 4;
                mma_ss(lead, t_s, qd + step, kd + step, hi, id_s, j > 0);
              }
              tc_commit_lead(lead, s_full + s);   // (the stream's threads give K's place back when they see it)
              if (k + 1 == tiles - 1) tc_commit_lead(lead, q_free);
            }
          }
          if (k >= 0 && ok) tc_commit_lead(lead, empty + v_slot);
        }
        if (tiles == 0) ok = warp_wait(ok, o_free, (item & 1) ^ 1, err);
        if (ok) tc_commit_lead(lead, o_done);
        turn += tiles;
        seq0 += 2 * n;
        pass(seq0);
      }
    } else {
      // ---- Q: a tile's tokens x G heads of one key head ----
      const uint32_t lead = elect_one();
      unsigned item = 0;
      Walk w;
      for (w.start(a, st); w.more(); w.next(a), ++item) {
        ok = warp_wait(ok, q_free, (item & 1) ^ 1, err);
        if (!ok) continue;
        const int both = w.dual(a) ? 2 : 1;
        mbar_expect_tx_lead(lead, q_full, both * a.rt * HD * 2);
        for (int x = 0; x < both; ++x)
#pragma unroll
          for (int panel = 0; panel < C::PANELS; ++panel)
            tma_load_4d(lead, smem_u32(smem + C::Q_OFF) + x * C::Q_TILE + panel * C::Q_PANEL, &tmq, smem_u32(q_full),
                        panel * (C::SW / 2), 0, w.kh, w.r.t0 + (2 * w.blk + x) * (a.block_tokens / 2));
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kStreamRegs));
    // ---- a stream: softmax, and the block's results; a thread a row ----
    const int s = (warp - 4) >> 2, r = tid & 127;
    const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);   // this warp's 32 TMEM lanes
    const uint32_t t_s = lanes + s * C::S_COL, t_o = lanes + C::O_COL + s * C::O_STEP;
    float2* xchg = reinterpret_cast<float2*>(smem + C::X_OFF);
    unsigned item = 0, turn = 0, seq0 = 0;
    struct Shared {   // a block that other CTAs have a part of
      int b, kh, blk, first, parts;
    } cut[2];
    int cuts = 0;
    Walk& w = reinterpret_cast<Walk*>(smem + C::WALK_OFF)[warp - 4];   // (the warp's; in registers it would not stay)
    if (lane == 0) w.start(a, st);
    __syncwarp();
    for (; w.more(); ++item) {
      const bool dual = w.dual(a);
      const int n = w.tiles, row = dual ? s * a.rt + r : r, here = min(a.rt, w.rows - (row - r));
      const bool mine = r < here;                                // this thread's row exists
      const bool active = (r & ~31) < here;                      // .. one of the warp's does
      const int tok = min(w.blk * 2 * a.rt + row, w.r.rows - 1) / a.G;
      const int seen_all = (int)min((long long)w.r.ctx + (a.mask ? 0 : w.blk * a.block_tokens + 1), (long long)a.cap);
      float m = -INFINITY, l = 0.f;
      const int tiles = dual ? n : (n - s + 1) / 2, ahead = k_lead(dual);
#pragma unroll 1
      for (int k = 0; k < tiles; ++k) {
        const int i = dual ? k : 2 * k + s, key0 = (w.tile0 + i) * kTile;
        const bool masked = key0 + kTile > seen_all;
        uint32_t see[4];
        if (__builtin_expect(masked && active, 0)) seen_keys(a, w.r, tok, key0, see);   // (under the product)
        ok = warp_wait(ok, s_full + s, (turn + k) & 1, err);
        tc_fence_after();
        if (r == 0 && ok) mbar_arrive(empty + (seq0 + seq_k(ahead, i)) % C::STAGES);
        uint32_t x[128];
        if (active) {
#pragma unroll
          for (int j = 0; j < 4; ++j) tmem_ld_32x32b_x32(t_s + 32 * j, *reinterpret_cast<uint32_t(*)[32]>(x + 32 * j));
          tmem_ld_wait128(x);
          if (__builtin_expect(masked, 0)) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (!(see[j] >> e & 1)) x[32 * j + e] = 0xff800000u;   // -infinity
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int j = 0; j < 64; ++j)
            mx[j & 3] = fmaxf(mx[j & 3], fmaxf(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1])));
          const float m_new = fmaxf(m, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.c - (VF16 ? kRaise : 0.f));
          const bool rise = mine && (m == -INFINITY ? m_new > m : m_new > m + kSlack);
          if (__builtin_expect(__any_sync(0xffffffffu, rise), 0)) {
            const float f = !rise ? 1.f : m == -INFINITY ? 0.f : exp2_fast(m - m_new);
            if (k > 0) {   // (O is at rest: S is complete, which was issued after the P V before)
#pragma unroll 1
              for (int c = 0; c < HD; c += 16) {
                uint32_t o[16];
                tmem_ld_32x32b_x16(t_o + c, o);
                tmem_ld_wait();
                float z[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) z[j] = __uint_as_float(o[j]) * f;
                tmem_st_32x32b_x16(t_o + c, z);
              }
            }
            l *= f;
            if (rise) m = m_new;
          }
        }
        // The streams' exponentials take turns, scheduler by scheduler (a warp of each): both at once would share one special
        // function unit and leave the tensor core to both streams' products at once after.
        if (dual && (s == 1 || k > 0)) named_bar_sync(4 + 4 * s + (warp & 3), 64);
        if (active) {
          const float base = m == -INFINITY ? 0.f : -m;
          const float2 c2 = make_float2(a.c, a.c), b2 = make_float2(base, base);
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 32 * h; j < 32 * h + 32; ++j) {
              float2 z = fma2(make_float2(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1])), c2, b2);
              z.x = exp2_fast(z.x), z.y = exp2_fast(z.y);
              sum[j & 1] = add2(sum[j & 1], z);
              x[j] = pack2(z.x, z.y, VF16);
            }
            tmem_st_32x32b_x32(t_s + 32 * h, x + 32 * h);
            if (h == 0 && !masked) {   // (masked: once the tile's V is seen to, below)
              tmem_st_wait();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(p_ready + 2 * s);
            }
            // (the second half's exponentials stay behind the first half's store)
            if (h == 0) hold64(x + 64);
          }
          sum[0] = add2(sum[0], sum[1]);
          l += sum[0].x + sum[0].y;
        }
        if (dual && (s == 0 || k + 1 < n)) named_bar_arrive(8 - 4 * s + (warp & 3), 64);
        if (active) tmem_st_wait();
        if (__builtin_expect(masked, 0)) {
          // V rows that some row of the block does not see: a NaN or infinity there would reach it as 0 x NaN.  They
          // become 0 in the tile (every one of them), and the rows that do see one get it back at the end.
          const unsigned seq = seq0 + seq_v(ahead, i, n), slot = seq % C::STAGES;
          ok = warp_wait(ok, full + slot, seq / C::STAGES & 1, err);   // (the place's copy before was seen with K's)
          clean_v<HD>(smem + slot * C::TILE, r, max(0, seen_all - key0), w.keys - key0, VF16, odd_v);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (masked || !active) mbar_arrive(p_ready + 2 * s);
          mbar_arrive(p_ready + 2 * s + 1);
        }
      }
      turn += tiles;
      // ---- the block's (or this part's) result ----
      float f0 = 1.f, f1 = 0.f, m_all = m, l_all = l;   // weights of the own stream's O, or of both streams' O
      if (!dual) {
        xchg[s * 128 + r] = make_float2(m, l);
        named_bar_sync(1, kStreamThreads);
        const float2 e0 = xchg[r], e1 = xchg[128 + r];
        named_bar_sync(1, kStreamThreads);
        m_all = fmaxf(e0.x, e1.x);
        f0 = e0.x == -INFINITY ? e0.y : exp2_fast(e0.x - m_all);   // (nothing seen: 0, or a NaN)
        f1 = e1.x == -INFINITY ? e1.y : exp2_fast(e1.x - m_all);
        l_all = (e0.x == -INFINITY ? e0.y : f0 * e0.y) + (e1.x == -INFINITY ? e1.y : f1 * e1.y);
      }
      ok = warp_wait(ok, o_done, item & 1, err);
      tc_fence_after();
      const bool whole = w.tile0 == 0 && n == w.all;
      const int slot = w.tile0 > 0 ? 0 : 1;
      float* part = part_of<HD>(a, blockIdx.x, slot);
      const float inv = whole ? (l_all == 0.f ? 0.f : 1.f / l_all) : 1.f;
      const int rg = w.blk * 2 * a.rt + row, t = w.r.t0 + tok, head = w.kh * a.G + (mine ? rg % a.G : 0);
      const int width = dual ? HD : HD / 2, c0 = dual ? 0 : s * width;   // this thread's columns
      if (active && ok) {
        const uint32_t o0 = lanes + C::O_COL + (dual ? s * C::O_STEP : 0), o1 = lanes + C::O_COL + C::O_STEP;
        uint16_t* out = a.out + (long long)t * a.out_stride + (long long)head * HD;
        float* prow = whole ? nullptr : part + row * HD;
        const float g0 = f0 * inv, g1 = f1 * inv;
#pragma unroll 1
        for (int c = c0; c < c0 + width; c += 16) {
          uint32_t y0[16], y1[16];
          tmem_ld_32x32b_x16(o0 + c, y0);
          tmem_ld_32x32b_x16(o1 + c, y1);   // (dual: with weight 0)
          tmem_ld_wait16(y0, y1);
          float y[16];
#pragma unroll
          for (int j = 0; j < 16; ++j)   // (a stream without tiles leaves its O as it was: a weight of 0 takes nothing from it)
            y[j] = (f0 == 0.f ? 0.f : __uint_as_float(y0[j]) * g0) + (f1 == 0.f ? 0.f : __uint_as_float(y1[j]) * g1);
          if (!mine) continue;
          if (whole) {
            uint32_t u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = pack2(y[2 * j], y[2 * j + 1], KF16);
            if (a.out32) {
              st_global_32(out + c, u);
            } else {
              reinterpret_cast<uint4*>(out + c)[0] = make_uint4(u[0], u[1], u[2], u[3]);
              reinterpret_cast<uint4*>(out + c)[1] = make_uint4(u[4], u[5], u[6], u[7]);
            }
          } else {
            st_global_32(prow + c, reinterpret_cast<const uint32_t(&)[8]>(y[0]));
            st_global_32(prow + c + 8, reinterpret_cast<const uint32_t(&)[8]>(y[8]));
          }
        }
        if (mine && *odd_v)
          add_odd_v<HD>(a, w.b, w.kh, tok, max(w.tile0 * kTile, seen_all), min(w.keys, (w.tile0 + n) * kTile), c0, c0 + width, out,
                        prow);
        if (mine && c0 == 0) {
          if (!whole) reinterpret_cast<float2*>(part + kBlock * HD)[row] = make_float2(m_all, l_all);
          else if (a.lse)
            a.lse[(long long)t * a.H + head] = l_all == 0.f ? -INFINITY : (m_all + log2f(l_all)) * 0.6931471805599453f;
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_free);
      if (!whole) {
        const int slack = block_slack(a, w.rows, st.most);
        const long long end = w.begin + w.cost + w.all;
        const auto border = [&](int cta) { return quotient(cta * st.units, st.ctas); };   // (before it is moved)
        Shared& x = cut[cuts++];
        int last = cta_of(end - 1, st);
        x.b = w.b, x.kh = w.kh, x.blk = w.blk, x.first = cta_of(w.begin + w.cost, st);
        if (const long long u = border(x.first + 1); x.first + 1 < st.ctas && u < end && u - w.begin <= slack) ++x.first;
        if (const long long u = border(last); u - w.begin > slack && end - u <= slack) --last;
        x.parts = last - x.first + 1;
        __threadfence();
        named_bar_sync(2 + s, 128);
        if (r == 0 && ok) asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(a.arrived + x.first) : "memory");
      }
      seq0 += 2 * n;
      __syncwarp();
      if (lane == 0) w.next(a);
      __syncwarp();
    }
    // ---- shares of the blocks that were cut ----
    for (int k = 0; k < cuts; ++k) {
      const Shared x = cut[k];
      if (tid == 128 && ok) ok = wait_count(a.arrived + x.first, 2 * x.parts, err);   // (one thread asks)
      ok = named_bar_and(1, kStreamThreads, ok);
      if (ok)
        merge_share<HD>(a, request(a, x.b), x.kh, x.blk, x.first, x.parts, blockIdx.x - x.first, tid - 128,
                        reinterpret_cast<float*>(smem + C::X_OFF));
      named_bar_sync(1, kStreamThreads);
      if (tid == 128 && ok && atomicAdd(a.done + x.first, 1) == x.parts - 1) {   // the last share: counters back to zero
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
  if (warp == 3) {
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

// A map of four dimensions, of 16-bit values, in boxes of up to 64 of the first.  Strides in elements.
atspeed_status map4(CUtensorMap* m, const void* base, int type, const int (&n)[4], const int64_t (&stride)[3],
                    const int (&box)[3]) {
  auto fn = encode_fn();
  if (!fn) return ATSPEED_E_CUDA;
  const int w = n[0] < 64 ? n[0] : 64;
  cuuint64_t dims[4], strides[3];
  cuuint32_t boxes[4] = {(cuuint32_t)w, (cuuint32_t)box[0], (cuuint32_t)box[1], (cuuint32_t)box[2]}, es[4] = {1, 1, 1, 1};
  for (int i = 0; i < 4; ++i) dims[i] = (cuuint64_t)n[i];
  // (the stride of a dimension of one entry is never used; the encoder wants a valid one)
  for (int i = 0; i < 3; ++i) strides[i] = (cuuint64_t)(n[i + 1] == 1 && stride[i] == 0 ? n[0] : stride[i]) * 2;
  const CUresult r = fn(m, type == ATSPEED_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
                        const_cast<void*>(base), dims, strides, boxes, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        w == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ATSPEED_OK : ATSPEED_E_ARG;
}
// [page][token][head][dimension] of a cache: boxes of the tokens of a page, or of half a page
atspeed_status page_map(CUtensorMap* m, const void* base, int type, const atspeed_kv_pages& c, const int64_t* stride) {
  return map4(m, base, type, {c.head_dim, c.page_size, c.n_kv_heads, c.n_pages}, {stride[1], stride[2], stride[0]},
              {c.page_size < kTile ? c.page_size : kTile, 1, 1});
}

template <int HD, bool KF16, bool VF16>
atspeed_status launch(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const TreeAttnArgs& a, int grid,
                      cudaStream_t st) {
  const auto kernel = tree_attention_kernel<HD, KF16, VF16>;
  static std::atomic<unsigned long long> done{0};
  if (smem_attr_once(done, kernel, Cfg<HD>::SMEM) != cudaSuccess) return ATSPEED_E_CUDA;
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
  return cudaLaunchKernelEx(&cfg, kernel, mq, mk, mv, a) == cudaSuccess ? ATSPEED_OK : ATSPEED_E_CUDA;
}
template <int HD>
atspeed_status launch(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const TreeAttnArgs& a, int grid,
                      cudaStream_t st) {
  if (a.k_f16) return launch<HD, true, true>(mq, mk, mv, a, grid, st);
  return a.v_f16 ? launch<HD, false, true>(mq, mk, mv, a, grid, st) : launch<HD, false, false>(mq, mk, mv, a, grid, st);
}

int sm_count() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  return gemm_grid_size(dev);
}

constexpr size_t kCounterBytes = ATSPEED_TREE_ATTENTION_COUNTER_BYTES;
static_assert(2 * kMaxCtas * sizeof(int) <= kCounterBytes, "the workspace's counters");

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
  const int G = n_heads / c.n_kv_heads;
  CUtensorMap mq, mk, mv;
  atspeed_status st = map4(&mq, d_q, c.k_type, {hd, G, c.n_kv_heads, T}, {hd, (int64_t)G * hd, q_stride}, {G, 1, 128 / G});
  if (st == ATSPEED_OK) st = page_map(&mk, c.d_k, c.k_type, c, c.k_stride);
  if (st == ATSPEED_OK) st = page_map(&mv, c.d_v, c.v_type, c, c.v_stride);
  if (st != ATSPEED_OK) return st;
  TreeAttnArgs a = {};
  a.v = static_cast<const uint16_t*>(c.d_v);
  for (int i = 0; i < 3; ++i) a.vs[i] = c.v_stride[i];
  a.out_stride = out_stride, a.rt = 128 / G * G, a.block_tokens = 2 * (128 / G);
  a.H = n_heads, a.Hkv = c.n_kv_heads, a.G = G, a.n = n_req, a.T = T, a.page_log = ps == 16 ? 4 : ps == 32 ? 5 : ps == 64 ? 6 : ps == 128 ? 7 : 8, a.page = ps, a.n_pages = c.n_pages;
  a.width = table_width, a.words = mask_words, a.cu_q = d_cu_q, a.ctx = d_ctx_len, a.table = d_block_table, a.mask = d_mask;
  const long long cap = (long long)table_width * ps;
  a.cap = (int)(cap < (1LL << 30) ? cap : 1LL << 30);
  a.c = scale * 1.4426950408889634f;
  a.out = static_cast<uint16_t*>(d_out), a.lse = d_lse;
  a.k_f16 = c.k_type == ATSPEED_F16, a.v_f16 = c.v_type == ATSPEED_F16;
  a.out32 = ((reinterpret_cast<uintptr_t>(d_out) | (uintptr_t)out_stride * 2) & 31) == 0;
  a.arrived = static_cast<int*>(d_ws), a.done = a.arrived + kMaxCtas;
  a.parts = static_cast<unsigned char*>(d_ws) + kCounterBytes;
  a.err = tree_attn_err_word();
  const int grid = sm_count();
  if (!a.err || grid <= 0 || grid > kMaxCtas) return ATSPEED_E_CUDA;
  if (hd == 32) return launch<32>(mq, mk, mv, a, grid, (cudaStream_t)stream);
  if (hd == 64) return launch<64>(mq, mk, mv, a, grid, (cudaStream_t)stream);
  return launch<128>(mq, mk, mv, a, grid, (cudaStream_t)stream);
}

}  // extern "C"
