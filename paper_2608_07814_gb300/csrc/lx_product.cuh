// The large matrix products of lx_linear and lx_head_loss, sm_103a tcgen05:
//   D [M][N] = sum_k A(m, k) B(n, k)      (bf16, or e4m3 where F8)
// in tiles of 256 x 256 that a pair of CTAs holds together (cta_group::2, M = N = 256):
// each CTA loads its 128 rows of A and half of B's 256, so an SM fetches 32 KiB for
// 128 x 256 x 64 products where a CTA by itself fetches 48.  The two operands may be stored
// along K (rows of D's row or column index, K contiguous) or along M / N (rows of K): the
// gradients read the activations, the weights and the gradient of the product as they are,
// without a transposed copy.
//
// One persistent pair an SM pair, 12 warps a CTA:
//   warp 0       asks for the operands' tiles (TMA, 128-byte swizzle, STAGES deep); the bytes
//                of both CTAs are counted by the even CTA's barrier;
//   warp 1       of the even CTA issues tcgen05.mma and commits stages and accumulators to
//                both CTAs; (of both) allocates 512 TMEM columns: two accumulators, so that
//                a tile's epilogue runs beside the next tile's products;
//   warps 4..11  epilogue: 32 rows x 64 columns at a time from TMEM, what the caller's MODE
//                makes of them, and TMA from a warp's buffers of shared memory to memory.
// Tiles are dealt in an order that keeps 16 rows of tiles together, so that what runs at the
// same time shares its operands in L2.  Every wait is bounded: when one gives up, the pair's
// tiles from there on are NaN, copies and products in flight are waited for, and TMEM is freed.
#pragma once

#include <algorithm>

#include "lx_rows.cuh"
#include "lx_tcgen05.cuh"

namespace lx {
namespace prod {

// A map of rows of `inner` bytes, ld bytes apart, in boxes of 128 bytes x box_rows rows
bool encode_bytes_2d(CUtensorMap* m, const void* base, long inner, long rows, long ld, int box_rows);

namespace {  // (each file that includes this has the kernels it launches)

using namespace tcg;

constexpr int BM = 256, BN = 256;      // a pair's tile
constexpr int KB = 128;                // bytes of K a stage: 64 bf16 or 128 e4m3
constexpr int A_BYTES = 128 * KB, STAGE = 2 * A_BYTES;
constexpr int EPI = 8, THREADS = 128 + 32 * EPI;
// Blocks of 32 rows x 64 columns leave a warp through buffers of 4 KiB (128-byte rows,
// 128-byte swizzle) by TMA: stores of 16 bytes a lane took 1.8 k cycles for 32 x 32, four
// times what the products of 64 inputs take.
constexpr int STG = 4096, PRM = 192;
constexpr int STG_LD = 80;             // rows TMA cannot take: 32 bf16, 16-byte pieces of 8 rows on distinct banks
constexpr int GROUP_M = 16, MAX_SLICES = 16;
constexpr int LEAVING = 5;  // blocks of K whose products take as long as a tile's way out (1.9 us)

// A CTA's words beside its barriers: whether one of its waits gave up, and whether one of the pair's
// did; the address of its TMEM; and, at its end, blocks of K that it asked for, blocks that were
// multiplied and sums that were committed (by the even CTA).
enum Word { LOST = 0, LOST_PAIR = 1, TMEM = 2, ASKED = 3, MADE = 4, SUMS = 5, WORDS = 6 };

enum Mode { LINEAR = 0, STATS = 1, DLOGIT = 2, GRAD = 3 };
enum Act { NONE = 0, RELU = 1, SILU = 2, GELU = 3 };

// What the stages and an epilogue warp's buffers make of an SM's shared memory.  DEEP: six stages and
// one buffer, else five and two, which a residual and the sums before the activation pass through.
// (8192 x 8192 x 2048: 155.6 us with six, 159.2 with five, 179.9 with four.  The gradients show no
// difference between six and five, not of short sums either, and the statistics none above five.)
template <int MODE, bool DEEP>
struct Cfg {
  static constexpr int NBUF = MODE == STATS ? 0 : DEEP ? 1 : 2;
  static constexpr int STAGES = MODE == STATS ? 5 : DEEP ? 6 : 5;
  static constexpr int PARAMS = MODE == LINEAR ? PRM : 0;
  static constexpr int BARS = 2 * STAGES + 5 + (MODE == LINEAR && !DEEP ? 2 * EPI : 0);
  static constexpr int SMEM = STAGES * STAGE + EPI * (NBUF * STG + PARAMS) + 8 * BARS + 4 * WORDS + 1024;
  static_assert(SMEM <= 227 * 1024, "fits an SM");
};

// One product of a launch.  Its tiles: slices (ranges of K) x tiles of N x tiles of M.
struct Problem {
  CUtensorMap a, b;  // maps of bytes: 128 x 128 boxes of an operand along K, 128 x 64 of one along M / N
  int a_mn, b_mn;    // stored along M / N
  int M, N, K;       // K in elements
  int slices;        // ranges of K side by side (into blocks, with `rows`: as slices_of has them)
  const int* rows;   // device count that bounds M (NULL: M), and
  const int* depth;  // one that bounds K
  // GRAD: bf16 (boxes of 128 bytes x 32 rows), or fp32 in blocks of 32 x 32, slice by slice
  CUtensorMap out;
  float* blocks;     // [slice][rows of tiles x 8][blocks of columns], a block's columns of 32 rows
  int add;           // to what the blocks hold
};

// What becomes of a sum of lx_linear: y = act(sum x_scale w_scale + bias) + residual
struct Epilogue {
  const float *x_scale, *w_scale;
  const __nv_bfloat16 *bias, *residual;
  __nv_bfloat16 *y, *pre;
  long ldr, ldy, ldp;
  int act;
  int unmet;  // test hook: the issuer first waits for what nothing fulfils
  unsigned long long wait_cycles;
};

struct Launch : Epilogue {
  Problem p[2];
  int n;
  // GRAD: columns' sums to be added up beside the products
  const float* db_part;
  int db_chunks, db_n;
  __nv_bfloat16* db;
  // LINEAR
  int tma_r, tma_y, tma_p;  // whether the residual's, y's and pre's rows suit TMA (boxes of 128 bytes x 32 rows):
  CUtensorMap map_r, map_y, map_p;
  // DLOGIT: compact rows' log-sum-exps (in units of log 2); STATS too: labels, and out of it the
  // label's logit, into DLOGIT its dz
  const float* lse2;
  const int* label;
  float* own;
  CUtensorMap map_dl;  // dz of the piece
  int v0;            // the first column's place in the vocabulary
  // STATS
  float2* part;      // [halves of tiles of N][part_ld]: a row's largest logit there, sum of exp
  long part_ld;
  float* keep;       // the logits in blocks of 32 x 32 (32 rows of each column), or NULL
  int keep_cols;     // blocks side by side
};

static __device__ __forceinline__ uint32_t mapa0(uint32_t addr) {  // the even CTA's
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
static __device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
static __device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A bounded wait (see mbar_wait) whose tries suspend the thread for up to 0.2 ms instead of
// polling: what the many waiting warps read of shared memory the products would have to wait for.
static __device__ __forceinline__ bool wait_quiet(uint32_t bar, uint32_t parity, volatile int* lost,
                                                  unsigned long long limit) {
  const unsigned long long t0 = clock64();
  while (true) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(200000u)
        : "memory");
    if (ok) return true;
    if (lost && *lost) return false;
    if (clock64() - t0 > limit) return false;
  }
}
// a word of shared memory of the pair's CTA
static __device__ __forceinline__ uint32_t get_word(const uint32_t* word, uint32_t rank) {
  uint32_t at, v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(word)), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
static __device__ __forceinline__ void set_word(uint32_t* word, uint32_t rank, uint32_t v) {
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(word)), "r"(rank));
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
}
static __device__ __forceinline__ void arrive_remote(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
static __device__ __forceinline__ void load_pair(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar)
      : "memory");
}
static __device__ __forceinline__ void commit_pair(uint32_t bar, uint16_t mask) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
      "h"(mask)
      : "memory");
}
template <bool F8>
static __device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  if constexpr (F8)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
// Descriptor of an operand stored along M / N: chunks of 64 elements (128 bytes, swizzled) x
// 64 rows of K, 8192 bytes apart (bits 16..29); 8 rows of K 1024 bytes apart (bits 32..45).
static __device__ __forceinline__ uint64_t desc_mn(uint32_t addr) {
  return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)(8192 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: fp32 accumulator (bits 4..5), A and B bf16 (1 at bits 7, 10) or
// e4m3 (0), stored along M (bit 15) / N (bit 16), N >> 3, M >> 4
__host__ __device__ constexpr uint32_t idesc(bool f8, int a_mn, int b_mn, int M, int N) {
  return (1u << 4) | (f8 ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// After a wait of the pair that gave up, one thread of each CTA, both CTAs being there until it is
// done: all copies asked for have landed, and all commits arrived, before shared memory and TMEM go
// away.  The roles stopped where they were, so this goes by their counts; no CTA is more than the
// stages ahead of the other, as a stage is asked for again once both halves of it were multiplied.  The
// bound is the default: what is waited for here is on its way and needs no one's part.
template <int STAGES>
static __device__ __noinline__ void settle(const uint32_t* words, uint32_t full0, uint32_t empty0, uint32_t tfull0,
                                           uint32_t rank) {
  const uint32_t even = get_word(words + ASKED, 0), odd = get_word(words + ASKED, 1), most = max(even, odd);
  const uint32_t made = get_word(words + MADE, 0), sums = get_word(words + SUMS, 0);
  if (rank == 0)  // (whose barriers count both CTAs' bytes)
    for (uint32_t j = most > STAGES ? most - STAGES : 0; j < most; ++j) {
      const uint32_t bar = full0 + 8 * (j % STAGES);
      if (j >= even)  // the odd CTA's half alone
        mbar_expect_tx(bar, STAGE);
      else if (j >= odd)  // the even one's: the other was expected, too
        asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(STAGE) : "memory");
      wait_quiet(bar, (j / STAGES) & 1, nullptr, kDefaultWaitCycles);
    }
  for (uint32_t j = made > STAGES ? made - STAGES : 0; j < made; ++j)
    wait_quiet(empty0 + 8 * (j % STAGES), (j / STAGES) & 1, nullptr, kDefaultWaitCycles);
  for (uint32_t j = sums > 2 ? sums - 2 : 0; j < sums; ++j)
    wait_quiet(tfull0 + 8 * (j & 1), (j >> 1) & 1, nullptr, kDefaultWaitCycles);
}

constexpr float LOG2E = 1.4426950408889634f;

// Activations.  A NaN stays one.
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The complementary error function by Abramowitz and Stegun 7.1.26: a polynomial in t = 1 / (1 + p x)
// times exp(-x^2), 1.5e-7 off at most (and some 2^-23 for the approximate reciprocal and exponential).
// That is a 2^-15 of bf16's step near 1; gelu's negative tail is |z| / 2 of it off, which relatively
// is 1.6e-3 at z = -5, 3.6e-3 at -6, 1e-2 at -8 and 3e-2 at -12 (1 + erf in fp32 is further off there).
// (With erff the epilogue took as long as 2500 inputs' products.)
// (a NaN stays one)
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float silu(float z) { return z * rcp(1.f + rows::ex2(-LOG2E * z)); }
// relu(z) - |z| times the function's tail, in pairs: 9 instructions a value, which bound the epilogue
// of 8-bit products of 2048 inputs.  |z| is held below 100, where the tail is 0.
__device__ __forceinline__ float2 gelu2(float2 z) {
  using rows::both;
  const float2 a = make_float2(fminf(fabsf(z.x), 100.f), fminf(fabsf(z.y), 100.f));
  const float2 q = rows::fma2(a, both(0.3275911f * 0.70710678f), both(1.f));
  const float2 t = make_float2(rcp(q.x), rcp(q.y));
  const float2 s = rows::mul2(rows::mul2(a, a), both(-0.5f * LOG2E));
  const float2 e = make_float2(rows::ex2(s.x), rows::ex2(s.y));
  float2 p = rows::fma2(both(0.5f * 1.061405429f), t, both(0.5f * -1.453152027f));
  p = rows::fma2(p, t, both(0.5f * 1.421413741f));
  p = rows::fma2(p, t, both(0.5f * -0.284496736f));
  p = rows::fma2(p, t, both(0.5f * 0.254829592f));
  p = rows::mul2(rows::mul2(p, t), e);
  return rows::fma2(make_float2(-a.x, -a.y), p, make_float2(max_nan(z.x, 0.f), max_nan(z.y, 0.f)));
}
template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N]) {
  if (act == RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = max_nan(v[i], 0.f);
  } else if (act == SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = silu(v[i]);
  } else if (act == GELU) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 y = gelu2(make_float2(v[i], v[i + 1]));
      v[i] = y.x, v[i + 1] = y.y;
    }
  }
}

struct Tile {
  int p, m0, n0, slice, kb0, nkb;
};

// Ranges of K of a product whose M is known on the device alone: as many more as there are
// fewer rows of tiles, in the same room
__host__ __device__ inline int slices_of(int slices, int M, int live) {
  const int mt = (M + BM - 1) / BM, lt = (live + BM - 1) / BM;
  const int n = lt > 0 ? slices * mt / lt : slices;
  return n < MAX_SLICES ? n : (slices > MAX_SLICES ? slices : MAX_SLICES);
}

// Sizes of the launch's products, as the device counts bound them, and the deal of their tiles:
// the first product's (whose sums are the longer) go round the pairs; the pairs that have one
// fewer are given `extra` of the second's, as many as take its time; the others go round again,
// from the last pair to the first.  (A plain round of both left 12 % of the pairs' time unused in
// the head's gradients of 4096 rows.)
struct Sizes {
  int M[2], mt[2], nt[2], kb[2], per[2], tiles[2];
  int pair, pairs, rest, extra, dealt;  // rest: pairs with one more of the first
  template <bool F8>
  __device__ void read(const Launch& P) {
    pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      tiles[i] = 0;
      per[i] = 1;
      if (i >= P.n) continue;
      const Problem& p = P.p[i];
      M[i] = p.rows ? min(*p.rows, p.M) : p.M;
      const int K = p.depth ? min(*p.depth, p.K) : p.K;
      const int slices = p.rows && p.blocks ? slices_of(p.slices, p.M, M[i]) : p.slices;
      mt[i] = (M[i] + BM - 1) / BM;
      nt[i] = (p.N + BN - 1) / BN;
      kb[i] = F8 ? (K + 127) / 128 : (K + 63) / 64;
      tiles[i] = mt[i] * nt[i] * slices;
      per[i] = (kb[i] + slices - 1) / slices;
    }
    rest = tiles[0] % pairs;
    extra = 0;
    if (rest) extra = min((per[0] + LEAVING / 2) / max(per[1], LEAVING), tiles[1] / (pairs - rest));
    dealt = extra * (pairs - rest);
  }
  // the pair's tile j
  __device__ bool at(int j, Tile& t) const {
    const int own = tiles[0] / pairs + (pair < rest);
    int i;
    if (j < own) {
      t.p = 0;
      i = pair + j * pairs;
    } else {
      t.p = 1;
      j -= own;
      const int mine = pair >= rest ? extra : 0;
      i = j < mine ? pair - rest + j * (pairs - rest) : dealt + pairs - 1 - pair + (j - mine) * pairs;
      if (i >= tiles[1]) return false;
    }
    const int m_n = t.p ? mt[1] : mt[0], n_n = t.p ? nt[1] : nt[0], kbs = t.p ? kb[1] : kb[0];
    const int run = t.p ? per[1] : per[0];
    t.slice = i / (m_n * n_n);
    i -= t.slice * m_n * n_n;
    const int g = i / (GROUP_M * n_n), gm = min(GROUP_M, m_n - g * GROUP_M);
    i -= g * GROUP_M * n_n;
    const int n = i / gm;
    t.m0 = (g * GROUP_M + i - n * gm) * BM;
    t.n0 = n * BN;
    t.kb0 = t.slice * run;
    t.nkb = max(0, min(run, kbs - t.kb0));
    return true;
  }
};

// 32 x 32 bf16 of a warp, a row a lane, through shared memory to rows of memory that TMA
// cannot take, a column a lane
__device__ __forceinline__ void put_rows(char* stg, const uint32_t* r, __nv_bfloat16* out, long ldo, int row0, int M,
                                         int col0, int N) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float* f = reinterpret_cast<const float*>(r) + 8 * j;
    *(uint4*)(stg + lane * STG_LD + 16 * j) =
        make_uint4(rows::to_bf2(make_float2(f[0], f[1])), rows::to_bf2(make_float2(f[2], f[3])),
                   rows::to_bf2(make_float2(f[4], f[5])), rows::to_bf2(make_float2(f[6], f[7])));
  }
  __syncwarp();
  if (col0 + lane < N) {
    const int n = min(32, M - row0);
    for (int i = 0; i < n; ++i)
      out[(long)(row0 + i) * ldo + col0 + lane] = *(const __nv_bfloat16*)(stg + i * STG_LD + 2 * lane);
  }
  __syncwarp();
}
// the other way, added to the lane's row
__device__ __forceinline__ void add_rows(char* stg, uint32_t* r, const __nv_bfloat16* in, long ld, int row0, int M,
                                         int col0, int N) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  if (col0 + lane < N) {
    const int n = min(32, M - row0);
#pragma unroll 8
    for (int i = 0; i < n; ++i)
      *(__nv_bfloat16*)(stg + i * STG_LD + 2 * lane) = in[(long)(row0 + i) * ld + col0 + lane];
  }
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint4 v = *(const uint4*)(stg + lane * STG_LD + 16 * j);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = rows::bf2(w[i]);
      r[8 * j + 2 * i] = __float_as_uint(__uint_as_float(r[8 * j + 2 * i]) + f.x);
      r[8 * j + 2 * i + 1] = __float_as_uint(__uint_as_float(r[8 * j + 2 * i + 1]) + f.y);
    }
  }
  __syncwarp();
}
// A lane's piece j (16 bytes) of its row in a buffer of 128-byte rows with the 128-byte swizzle
__device__ __forceinline__ uint4* piece(char* buf, int j) {
  const int lane = threadIdx.x & 31;
  return (uint4*)(buf + lane * 128 + ((j ^ (lane & 7)) << 4));
}
// 32 rows x 64 columns, a row a lane, by TMA; the buffer is free
__device__ __forceinline__ void put_box(char* buf, const uint32_t (&r)[64], const CUtensorMap* map, int col0, int row0) {
  const float* f = reinterpret_cast<const float*>(r);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    *piece(buf, j) = make_uint4(
        rows::to_bf2(make_float2(f[8 * j], f[8 * j + 1])), rows::to_bf2(make_float2(f[8 * j + 2], f[8 * j + 3])),
        rows::to_bf2(make_float2(f[8 * j + 4], f[8 * j + 5])), rows::to_bf2(make_float2(f[8 * j + 6], f[8 * j + 7])));
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if ((threadIdx.x & 31) == 0) {
    tma_store_2d(map, 2 * col0, row0, smem_u32(buf));
    bulk_commit();
  }
}
// at most N of the warp's boxes are still being read
template <int N>
__device__ __forceinline__ void box_wait() {
  if ((threadIdx.x & 31) == 0) bulk_wait_read<N>();
  __syncwarp();
}

// sum of a column's parts: 8 ranges of them, then those in order
__device__ __forceinline__ float column_sum(const float* part, int chunks, int n, int c) {
  const int per = (chunks + 7) / 8;
  float v = 0.f;
  for (int w = 0; w < 8; ++w) {
    float s = 0.f;
#pragma unroll 8
    for (int i = w * per; i < min(chunks, (w + 1) * per); ++i) s += part[(long)i * n + c];
    v += s;
  }
  return v;
}

// The tensor core cuts a running sum off at every instruction (16 terms, 32 of e4m3): a sum of
// 2048 is 1e-6 to 4e-6 of itself short.  That is lost in a bf16 output, but not in a loss: the logits'
// statistics are taken of sums in parts of 1024 terms (16 blocks of K), each in an accumulator of
// its own, added as fp32 on their way out.  (Losses were 1e-6 off, at 2560 terms 1.3e-6, and are
// 3e-7 to 6e-7; it costs these tiles 3 %.  In the gradients' tiles the registers for it cost 10 to 50 %.)
// The logits that become dz are summed in the same parts: they are those whose log-sum-exp is subtracted,
// to the bit, and a row's dz adds up to 0.  (Summed in one accumulator, all of a row's are too small alike:
// its dz added up to 0.017 for 4096 inputs and logits that share a part of 2000.)
template <int MODE, bool F8, bool DEEP>
__global__ void __launch_bounds__(THREADS, 1) k_product(const __grid_constant__ Launch P) {
  using C = Cfg<MODE, DEEP>;
  constexpr int STAGES = C::STAGES, NBUF = C::NBUF;
  constexpr bool PASS = MODE == LINEAR && !DEEP;  // takes a residual and keeps the sums
  constexpr bool PARTS = MODE == STATS || MODE == DLOGIT;
  constexpr int PART = PARTS ? 16 : 1 << 30;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  char* staged = reinterpret_cast<char*>(smem + STAGES * STAGE);
  uint64_t* bars = reinterpret_cast<uint64_t*>(staged + EPI * (NBUF * STG + C::PARAMS));
  const uint32_t base = smem_u32(smem), full0 = smem_u32(bars), empty0 = full0 + 8 * STAGES;
  const uint32_t tfull0 = empty0 + 8 * STAGES, tempty0 = tfull0 + 16, never = tempty0 + 16, res0 = never + 8;
  uint32_t* words = reinterpret_cast<uint32_t*>(bars + C::BARS);
  volatile int* lost = reinterpret_cast<volatile int*>(words + LOST);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full0 + 8 * s, 1);   // the even CTA's: its producer, and both CTAs' bytes
      mbar_init(empty0 + 8 * s, 1);  // a commit
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(tfull0 + 8 * b, 1);             // a commit
      mbar_init(tempty0 + 8 * b, 2 * EPI);      // the even CTA's: both CTAs' epilogue warps
    }
    mbar_init(never, 1);
    if (PASS)
      for (int i = 0; i < 2 * EPI; ++i) mbar_init(res0 + 8 * i, 1);
    words[LOST] = words[LOST_PAIR] = words[ASKED] = words[MADE] = words[SUMS] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(words + TMEM)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  Sizes S;
  S.read<F8>(P);
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers are there
  tc_fence_after();
  const uint32_t tmem = words[TMEM];

  Tile t;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int i = 0; ok && S.at(i, t); ++i) {
        const Problem& p = P.p[t.p];
        const int m = t.m0 + 128 * (int)rank, n = t.n0 + 128 * (int)rank;
        for (int k = 0; k < t.nkb; ++k, ++it) {
          const uint32_t s = it % STAGES;
          if (!wait_quiet(empty0 + 8 * s, ((it / STAGES) & 1) ^ 1, lost, P.wait_cycles)) {
            ok = false;
            break;
          }
          if (rank == 0) mbar_expect_tx(full0 + 8 * s, 2 * STAGE);
          const uint32_t bar = mapa0(full0 + 8 * s), as = base + s * STAGE, bs = as + A_BYTES;
          const int kb = t.kb0 + k;
          if (p.a_mn) {
            load_pair(as, &p.a, 2 * m, 64 * kb, bar);
            load_pair(as + 8192, &p.a, 2 * m + 128, 64 * kb, bar);
          } else {
            load_pair(as, &p.a, KB * kb, m, bar);
          }
          if (p.b_mn) {
            load_pair(bs, &p.b, 2 * n, 64 * kb, bar);
            load_pair(bs + 8192, &p.b, 2 * n + 128, 64 * kb, bar);
          } else {
            load_pair(bs, &p.b, KB * kb, n, bar);
          }
        }
      }
      // the commits of the last stages have arrived before the CTA may end
      for (uint32_t j = it > STAGES ? it - STAGES : 0; ok && j < it; ++j)
        ok = wait_quiet(empty0 + 8 * (j % STAGES), (j / STAGES) & 1, lost, P.wait_cycles);
      if (!ok) *lost = 1;
      words[ASKED] = it;
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      uint32_t it = 0, nt = 0;
      bool ok = !P.unmet || wait_quiet(never, 0, lost, P.wait_cycles);
      for (int i = 0; ok && S.at(i, t); ++i) {
        if (t.nkb == 0) continue;
        const Problem& p = P.p[t.p];
        const uint32_t id = idesc(F8, p.a_mn, p.b_mn, BM, BN);
        uint32_t d = tmem;
        for (int k = 0; k < t.nkb; ++k, ++it) {
          const uint32_t s = it % STAGES;
          if (k % PART == 0) {  // an accumulator for the next part of the sum
            if (k) commit_pair(tfull0 + 8 * (nt++ & 1), 3);
            ok = wait_quiet(tempty0 + 8 * (nt & 1), ((nt >> 1) & 1) ^ 1, lost, P.wait_cycles);
            if (!ok) break;
            tc_fence_after();
            d = tmem + (nt & 1) * BN;
          }
          ok = wait_quiet(full0 + 8 * s, (it / STAGES) & 1, lost, P.wait_cycles);
          if (!ok) break;
          tc_fence_after();
          const uint32_t as = base + s * STAGE, bs = as + A_BYTES;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint64_t da = p.a_mn ? desc_mn(as + 2048 * j) : smem_desc(as + 32 * j);
            const uint64_t db = p.b_mn ? desc_mn(bs + 2048 * j) : smem_desc(bs + 32 * j);
            mma_pair<F8>(d, da, db, id, k % PART != 0 || j != 0 ? 1u : 0u);
          }
          commit_pair(empty0 + 8 * s, 3);
        }
        if (ok) commit_pair(tfull0 + 8 * (nt++ & 1), 3);
      }
      if (!ok) *lost = 1;
      words[MADE] = it;
      words[SUMS] = nt;
    }
  } else if (MODE == GRAD && warp < 4) {
    for (int c = (blockIdx.x * 2 + warp - 2) * 32 + lane; c < P.db_n; c += gridDim.x * 64)
      P.db[c] = __float2bfloat16_rn(column_sum(P.db_part, P.db_chunks, P.db_n, c));
  } else if (warp >= 4) {
    const int q = warp & 3, half = (warp - 4) >> 2;
    char* stg = staged + (warp - 4) * NBUF * STG;
    float* prm = reinterpret_cast<float*>(staged + EPI * NBUF * STG + (warp - 4) * C::PARAMS);  // scales, then the bias
    __nv_bfloat16* prm_b = reinterpret_cast<__nv_bfloat16*>(prm + 32);
    const uint32_t res = res0 + 16 * (warp - 4);
    uint32_t res_turn = 0;  // bit j: phase of buffer j's barrier
    const float nan = __int_as_float(0x7fc00000);
    uint32_t nt = 0;
    int ok = 1, last = -1;  // the buffer that the last box left from
    auto box_free = [&](int j) {
      if (NBUF < 2 || last == j) box_wait<0>();
      else box_wait<1>();
      last = j;
    };
    for (int i = 0; S.at(i, t); ++i) {
      const Problem& p = P.p[t.p];
      const int M = t.p ? S.M[1] : S.M[0];
      const int row0 = t.m0 + 128 * (int)rank + 32 * q, row = row0 + lane;
      // dz has rows of zeros behind the last: whole tiles
      const bool on = row0 < (MODE == DLOGIT ? p.M : M);
      // the residual's block j by TMA into its buffer, once what left it has been read
      auto fetch = [&](int j) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        box_wait<0>();
        if (lane == 0) {
          mbar_expect_tx(res + 8 * j, STG);
          tma_load_2d(smem_u32(stg + j * STG), &P.map_r, 2 * (t.n0 + 128 * half + 64 * j), row0, res + 8 * j);
        }
      };
      const bool ahead = PASS && P.tma_r && on;
      if (ahead) {
        if (t.n0 + 128 * half < p.N) fetch(0);
        if (!P.pre && t.n0 + 128 * half + 64 < p.N) fetch(1);
      }
      // what the tile needs besides its sums, on the way while those are formed: the row's, and
      // the scales and biases of the columns 32 h + lane
      int label = -1;
      float lse2 = 0.f, own = 0.f, xs = 1.f, col_s[4];
      __nv_bfloat16 col_b[4];
      if (MODE == STATS && row < M) label = P.label[row];
      if (MODE == DLOGIT && row < M) label = P.label[row] - P.v0, lse2 = P.lse2[row], own = P.own[row];
      if (MODE == LINEAR) {
        if (F8 && row < M) xs = P.x_scale[row];
        if (F8 || P.bias)
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            const int col = t.n0 + 128 * half + 32 * h + lane;
            col_b[h] = P.bias && col < p.N ? P.bias[col] : __float2bfloat16_rn(0.f);
            if (F8) col_s[h] = col < p.N ? P.w_scale[col] : 0.f;
          }
      }
      // the next part of the sum is there
      auto arrived = [&] {
        if (ok && lane == 0) {
          ok = wait_quiet(tfull0 + 8 * (nt & 1), (nt >> 1) & 1, lost, P.wait_cycles) ? 1 : 0;
          if (!ok) *lost = 1;
        }
        ok = __shfl_sync(0xffffffffu, ok, 0);
        tc_fence_after();
      };
      // it has been read: its accumulator may take the next part but one
      auto release = [&] {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_remote(mapa0(tempty0 + 8 * (nt & 1)));
      };
      const uint32_t mine = tmem + ((uint32_t)(32 * q) << 16) + 128 * half;
      float best = -INFINITY, total = 0.f;  // STATS
      // 64 columns of the warp's rows
      auto leave = [&](int j, uint32_t(&r)[64]) {
        const int col0 = t.n0 + 128 * half + 64 * j;
        char* buf = stg + (NBUF == 2 ? j * STG : 0);
        if (col0 >= p.N || !on) return;
        if constexpr (MODE == STATS) {
          const int n = min(64, p.N - col0), at_label = label - col0;
          if (at_label >= 0 && at_label < n) {
            float z = 0.f;
#pragma unroll
            for (int e = 0; e < 64; ++e)
              if (at_label == e) z = __uint_as_float(r[e]);
            P.own[row] = z;
          }
          __syncwarp();
          if (P.keep) {
            float* o = P.keep + ((long)(row0 / 32) * P.keep_cols + col0 / 32) * 1024 + lane;
#pragma unroll
            for (int e = 0; e < 64; ++e) o[32 * e] = __uint_as_float(r[e]);  // (keep_cols is even)
          }
          if (n < 64)
#pragma unroll
            for (int e = 0; e < 64; ++e)
              if (e >= n) r[e] = 0xff800000u;  // -inf
          float m = best;
#pragma unroll
          for (int e = 0; e < 64; ++e) m = fmaxf(m, __uint_as_float(r[e]));
          // exponentials of what is left of the largest value, whose own is then 1 and no other above
          const float2 at = rows::both(m == -INFINITY ? 0.f : -m);  // (a row of -inf so far)
          float s0 = total * rows::ex2((best + at.x) * LOG2E), s1 = 0.f;
#pragma unroll
          for (int e = 0; e < 64; e += 2) {
            const float2 x = rows::mul2(rows::add2(make_float2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])), at),
                                        rows::both(LOG2E));
            s0 += rows::ex2(x.x);
            s1 += rows::ex2(x.y);
          }
          total = s0 + s1;
          best = m;
        } else if constexpr (MODE == DLOGIT) {
          // rounded to bf16 as the tensor cores take it: 2^-9 of each term of the gradients' fp32 sums
          const int at = label - col0;
#pragma unroll
          for (int e = 0; e < 64; ++e) {
            const float d = at == e ? own : rows::ex2(fmaf(__uint_as_float(r[e]), LOG2E, -lse2));
            r[e] = row < M ? __float_as_uint(d) : 0u;
          }
          box_free(j);
          put_box(buf, r, &P.map_dl, col0, row0);
        } else if constexpr (MODE == GRAD) {
          if (p.blocks) {
            const int ncb = (p.N + 31) / 32;
            float* o = p.blocks + (((long)t.slice * ((M + BM - 1) / BM * (BM / 32)) + row0 / 32) * ncb + col0 / 32) * 1024 + lane;
            const int n = min(2, ncb - col0 / 32);
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (h < n) {
                if (p.add) {
#pragma unroll
                  for (int e = 32 * h; e < 32 * h + 32; ++e)
                    r[e] = __float_as_uint(o[32 * e] + __uint_as_float(r[e]));
                }
#pragma unroll
                for (int e = 32 * h; e < 32 * h + 32; ++e) o[32 * e] = __uint_as_float(r[e]);
              }
          } else {
            box_free(j);
            put_box(buf, r, &p.out, col0, row0);
          }
        } else {
          if (PASS && ahead && P.pre && j == 1) fetch(1);
          // TMA stores whole pieces of 16 bytes: a last block that ends inside one goes by columns
          const bool whole = col0 + 64 <= p.N || p.N % 8 == 0;
          // the columns' scale and bias, handed to all lanes
          if (F8 || P.bias) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              __syncwarp();
              prm_b[lane] = j ? col_b[2 + h] : col_b[h];
              if (F8) prm[lane] = j ? col_s[2 + h] : col_s[h];
              __syncwarp();
#pragma unroll
              for (int e = 0; e < 32; e += 4) {
                const uint2 w = *(const uint2*)(prm_b + e);
                const float2 b0 = rows::bf2(w.x), b1 = rows::bf2(w.y);
                float4 s = make_float4(1.f, 1.f, 1.f, 1.f);
                if (F8) {
                  s = *(const float4*)(prm + e);
                  s.x *= xs, s.y *= xs, s.z *= xs, s.w *= xs;
                }
                uint32_t* z = r + 32 * h + e;
                z[0] = __float_as_uint(fmaf(__uint_as_float(z[0]), s.x, b0.x));
                z[1] = __float_as_uint(fmaf(__uint_as_float(z[1]), s.y, b0.y));
                z[2] = __float_as_uint(fmaf(__uint_as_float(z[2]), s.z, b1.x));
                z[3] = __float_as_uint(fmaf(__uint_as_float(z[3]), s.w, b1.y));
              }
            }
          }
          if (PASS && P.pre) {  // through the other buffer
            box_wait<0>();
            if (P.tma_p && whole) {
              put_box(stg + (j ^ 1) * STG, r, &P.map_p, col0, row0);
            } else {
              for (int h = 0; h < 2; ++h)
                put_rows(stg + (j ^ 1) * STG, r + 32 * h, P.pre, P.ldp, row0, M, col0 + 32 * h, p.N);
            }
          }
          activate(P.act, reinterpret_cast<float(&)[64]>(r));
          if (PASS && P.residual) {
            if (P.tma_r) {
              int got = 1;
              if (lane == 0)
                got = wait_quiet(res + 8 * j, (res_turn >> j) & 1, nullptr, kDefaultWaitCycles);  // (it is on its way)
              got = __shfl_sync(0xffffffffu, got, 0);
              res_turn ^= 1u << j;
              if (!got) {
                ok = 0;
                *lost = 1;
              }
              __syncwarp();
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const uint4 v = *piece(buf, k);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                  const float2 f = rows::bf2(w[u]);
                  r[8 * k + 2 * u] = __float_as_uint(got ? __uint_as_float(r[8 * k + 2 * u]) + f.x : nan);
                  r[8 * k + 2 * u + 1] = __float_as_uint(got ? __uint_as_float(r[8 * k + 2 * u + 1]) + f.y : nan);
                }
              }
            } else {
              box_wait<0>();
#pragma unroll
              for (int h = 0; h < 2; ++h) add_rows(buf, r + 32 * h, P.residual, P.ldr, row0, M, col0 + 32 * h, p.N);
            }
          }
          if (P.tma_y && whole) {
            if (!PASS || (!P.pre && !ahead)) box_free(j);  // (else the buffer has been waited for)
            put_box(buf, r, &P.map_y, col0, row0);
          } else {
            box_wait<0>();
#pragma unroll
            for (int h = 0; h < 2; ++h) put_rows(buf, r + 32 * h, P.y, P.ldy, row0, M, col0 + 32 * h, p.N);
          }
        }
      };
      if constexpr (PARTS) {
        uint32_t r[2][64];
        for (int k = 0; k < t.nkb; k += PART, ++nt) {
          arrived();
          if (!ok) continue;
          const uint32_t at = mine + (nt & 1) * BN;
          if (k == 0) {
#pragma unroll
            for (int h = 0; h < 4; ++h)
              tc_ld32_async(at + 32 * h, *reinterpret_cast<uint32_t(*)[32]>(&r[h / 2][32 * (h & 1)]));
            tc_wait_ld();
          } else {
#pragma unroll
            for (int h = 0; h < 8; ++h) {
              uint32_t s[16];
              tc_ld16_async(at + 16 * h, s);
              tc_wait_ld();
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                uint32_t& v = r[h / 4][16 * (h & 3) + e];
                v = __float_as_uint(__uint_as_float(v) + __uint_as_float(s[e]));
              }
            }
          }
          release();
        }
        if (t.nkb == 0 || !ok) {
#pragma unroll
          for (int e = 0; e < 64; ++e) r[0][e] = r[1][e] = ok ? 0u : __float_as_uint(nan);
        }
        leave(0, r[0]);
        leave(1, r[1]);
      } else {
        if (t.nkb > 0) arrived();
#pragma unroll 1
        for (int j = 0; j < 2; ++j) {
          uint32_t r[64];
          __syncwarp();
          if (t.nkb > 0 && ok) {
            const uint32_t at = mine + (nt & 1) * BN + 64 * j;
            tc_ld32_async(at, *reinterpret_cast<uint32_t(*)[32]>(r));
            tc_ld32_async(at + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
            tc_wait_ld();
            if (j == 1) release();
          } else {
#pragma unroll
            for (int e = 0; e < 64; ++e) r[e] = ok ? 0u : __float_as_uint(nan);
          }
          leave(j, r);
        }
        if (t.nkb > 0) ++nt;
      }
      if (MODE == STATS && row < M && t.n0 + 128 * half < p.N)
        P.part[(long)(t.n0 / 128 + half) * P.part_ld + row] = make_float2(ok ? best : nan, total);
    }
    if (lane == 0) bulk_wait_all();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *lost) set_word(words + LOST_PAIR, 0, 1), set_word(words + LOST_PAIR, 1, 1);
  __syncwarp();
  cluster_sync();
  if (*(volatile uint32_t*)(words + LOST_PAIR)) {  // in both CTAs
    if (threadIdx.x == 0) settle<STAGES>(words, full0, empty0, tfull0, rank);
    __syncwarp();
    cluster_sync();
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// A launch that may start while the one before it in the stream ends: its kernel waits for
// that (pdl_wait) before it reads or writes anything
template <typename... KArgs, typename... Args>
lx_status launch_after(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t st,
                       const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  LX_CUDA(cudaLaunchKernelEx(&cfg, kern, args...));
  return LX_OK;
}

// A product from its fp32 blocks: the slices in their order, rounded once, each row to its
// place.  A CTA a block, a warp four of its columns.
struct Join {
  const float* blocks;
  int M, N, slices;   // as the product's
  const int* rows;    // device count that bounds M, or NULL
  const int* place;   // a row's place, or NULL: itself,
  const float* scale; // and factor, or NULL: 1
  __nv_bfloat16* out; // rows of N (a multiple of 8)
  int rest;           // so many rows on is what is added to a row of the first 32, or 0
};
__global__ void __launch_bounds__(256) k_join(const __grid_constant__ Join A) {
  __shared__ __nv_bfloat16 stage[32][40];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n = A.rows ? min(*A.rows, A.M) : A.M, slices = A.rows ? slices_of(A.slices, A.M, n) : A.slices;
  const int rb = blockIdx.x, cb = blockIdx.y, ncb = gridDim.y;
  if (rb * 32 >= n) return;
  const long slice = (long)((n + BM - 1) / BM * (BM / 32)) * ncb * 1024;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  const float* b = A.blocks + ((long)rb * ncb + cb) * 1024 + 128 * warp + lane;
#pragma unroll 4
  for (int s = 0; s < slices; ++s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += b[s * slice + 32 * e];
  }
  if (A.rest) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += __shfl_down_sync(0xffffffffu, v[e], A.rest);
  }
  const float f = A.scale && rb * 32 + lane < n ? A.scale[rb * 32 + lane] : 1.f;
  *(uint2*)&stage[lane][4 * warp] = make_uint2(rows::to_bf2(make_float2(v[0] * f, v[1] * f)),
                                               rows::to_bf2(make_float2(v[2] * f, v[3] * f)));
  __syncthreads();
  const int r = threadIdx.x / 4, c = 8 * (threadIdx.x % 4), row = rb * 32 + r;
  if (threadIdx.x < 128 && row < n && cb * 32 + c < A.N)
    *(uint4*)(A.out + (long)(A.place ? A.place[row] : row) * A.N + cb * 32 + c) = *(const uint4*)&stage[r][c];
}
inline lx_status launch_join(const Join& J, cudaStream_t st) {
  return launch_after(k_join, dim3((J.M + 31) / 32, (J.N + 31) / 32), dim3(256), 0, 1, st, J);
}
// floats of a product's blocks
inline size_t block_floats(long M, long N, int slices) {
  return (size_t)slices * ((M + BM - 1) / BM * (BM / 32)) * ((N + 31) / 32) * 1024;
}

// Operand along K: rows x K elements of es bytes, ld elements apart; along M / N: K rows
inline bool operand(CUtensorMap* m, const void* base, long inner, long outer, long ld, int es, bool mn) {
  return encode_bytes_2d(m, base, inner * es, outer, ld * es, mn ? 64 : 128);
}

// bf16 rows written (or read) in boxes of 128 bytes x 32 rows, where TMA can
inline bool boxes(CUtensorMap* m, const void* base, long cols, long rows_, long ld) {
  return rows::aligned(base, 16) && ld % 8 == 0 && ld < (1L << 31) && encode_bytes_2d(m, base, 2 * cols, rows_, 2 * ld, 32);
}

inline long tiles_of(const Problem& p) {
  return (long)((p.M + BM - 1) / BM) * ((p.N + BN - 1) / BN) * p.slices;
}

template <int MODE, bool F8, bool DEEP>
lx_status launch_as(const Launch& P, unsigned pairs, cudaStream_t st) {
  static bool cap[64] = {};
  int dev = 0;
  LX_CUDA(cudaGetDevice(&dev));
  LX_CUDA(smem_cap_once((const void*)k_product<MODE, F8, DEEP>, Cfg<MODE, DEEP>::SMEM, dev, cap));
  return launch_after(k_product<MODE, F8, DEEP>, dim3(2 * pairs), dim3(THREADS), Cfg<MODE, DEEP>::SMEM, 2, st, P);
}

template <int MODE, bool F8>
lx_status launch_product(const Launch& P, cudaStream_t st) {
  long tiles = 0;
  for (int i = 0; i < P.n; ++i) tiles += tiles_of(P.p[i]);
  if (tiles == 0) return LX_OK;
  const unsigned pairs = (unsigned)std::min<long>(tiles, rows::SMS / 2);
  if constexpr (MODE == LINEAR)
    if (P.residual || P.pre) return launch_as<MODE, F8, false>(P, pairs, st);
  return launch_as<MODE, F8, true>(P, pairs, st);
}

}  // namespace
}  // namespace prod
}  // namespace lx
