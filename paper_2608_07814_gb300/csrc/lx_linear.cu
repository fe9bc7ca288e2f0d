// A dense product with its epilogue, and its gradients (lx_linear, lx_linear_backward):
//   z = x W^T (x_scale w_scale) + b,  y = act(z) + residual
//   dz = dy act'(z),  dx = dz W,  dW = dz^T x,  db = sum_t dz
// Many tokens are bound by the tensor cores and run as tiles of 256 x 256 (lx_product.cuh).
// Few tokens are bound by reading W: k_linear_few holds 128 rows of W as the 128 rows of the
// tensor core's tile and up to 256 tokens as its columns, and splits K over the CTAs of a
// cluster, so that a product of few outputs still reads W with every SM; the CTAs' partial
// sums meet in shared memory, in the cluster's order, and the epilogue follows in the same launch.
#include "lx_product.cuh"

namespace lx {
namespace {

using namespace rows;
using namespace prod;

// ---------------------------------------------------------------------------
// few tokens
// ---------------------------------------------------------------------------
constexpr int FEW_THREADS = 256, FEW_SPLIT = 8, FEW_T = 256;

struct Few {
  CUtensorMap w, x;  // boxes of 128 bytes x 128 rows, and x tn rows
  int T, N, nkb, per;  // blocks of K: all, a CTA's
  int tn, stages, cols;  // tokens of a tile (a multiple of 16), TMEM columns
  int vec;           // four outputs at a time
  Epilogue e;
};

template <bool F8>
static __device__ __forceinline__ void mma_one(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t acc) {
  if constexpr (F8)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(id), "r"(acc)
        : "memory");
  else
    tc_mma(d, a, b, id, acc);
}

static __device__ __forceinline__ float4 ld_cluster(uint32_t addr, uint32_t rank) {
  uint32_t at;
  float4 v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(at)
               : "memory");
  return v;
}

template <bool F8>
__global__ void __launch_bounds__(FEW_THREADS, 2) k_linear_few(const __grid_constant__ Few P) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars[2 * 16 + 1];
  __shared__ uint32_t tmem_s;
  __shared__ int lost_s;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  volatile int* lost = &lost_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(smem), full0 = smem_u32(bars), empty0 = full0 + 8 * 16, done = empty0 + 8 * 16;
  const uint32_t stage = A_BYTES + P.tn * KB;
  const int splits = gridDim.x, rank = blockIdx.x, n0 = blockIdx.y * 128, t0 = blockIdx.z * P.tn;
  const int kb0 = rank * P.per, nkb = max(0, min(P.per, P.nkb - kb0));
  if (threadIdx.x == 0) {
    for (int s = 0; s < P.stages; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, 1);
    }
    mbar_init(done, 1);
    *lost = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)),
                 "r"(P.cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_s;
  uint32_t issued = 0;
  if (warp == 0) {
    if (lane == 0)
      for (int i = 0; i < nkb; ++i) {
        const uint32_t s = i % P.stages, bar = full0 + 8 * s, as = base + s * stage;
        if (!wait_quiet(empty0 + 8 * s, ((i / P.stages) & 1) ^ 1, lost, P.e.wait_cycles)) {
          *lost = 1;
          break;
        }
        mbar_expect_tx(bar, stage);
        tma_load_2d(as, &P.w, KB * (kb0 + i), n0, bar);
        tma_load_2d(as + A_BYTES, &P.x, KB * (kb0 + i), t0, bar);
        issued = i + 1;
      }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t id = idesc(F8, 0, 0, 128, P.tn);
      bool ok = !P.e.unmet || wait_quiet(done, 0, lost, P.e.wait_cycles);
      for (int i = 0; ok && i < nkb; ++i) {
        const uint32_t s = i % P.stages, as = base + s * stage, bs = as + A_BYTES;
        if (!wait_quiet(full0 + 8 * s, (i / P.stages) & 1, lost, P.e.wait_cycles)) {
          ok = false;
          break;
        }
        tc_fence_after();
#pragma unroll
        for (int j = 0; j < 4; ++j)
          mma_one<F8>(tmem, smem_desc(as + 32 * j), smem_desc(bs + 32 * j), id, (i | j) != 0 ? 1u : 0u);
        tc_commit(empty0 + 8 * s);
      }
      if (!ok) *lost = 1;
      tc_commit(done);  // also on the way out: no product is in flight when TMEM is freed
    }
    __syncwarp();
  }
  // every warp: the sums into shared memory (the stages are free: every product has been
  // made), a token's 128 outputs a row; warp w reads TMEM lanes 32 (w % 4) ..
  int ok = 1;
  if (lane == 0) {
    ok = wait_quiet(done, 0, nullptr, 2 * P.e.wait_cycles) ? 1 : 0;  // (the issuer may have waited for the bound)
    if (!ok) {
      *lost = 1;
      wait_quiet(done, 0, nullptr, kDefaultWaitCycles);  // no product is in flight from here on
    } else if (*lost) {
      ok = 0;
    }
  }
  ok = __shfl_sync(0xffffffffu, ok, 0);
  tc_fence_after();
  if (!ok && warp == 0 && lane == 0) {
    // copies in flight land before the sums take their place
    const uint32_t first = issued > (uint32_t)P.stages ? issued - P.stages : 0;
    for (uint32_t j = first; j < issued; ++j)
      wait_quiet(full0 + 8 * (j % P.stages), (j / P.stages) & 1, nullptr, kDefaultWaitCycles);
  }
  __syncthreads();
  float* part = reinterpret_cast<float*>(smem);
  const int q = warp & 3, T = min(P.tn, P.T - t0);
  for (int c = (warp >> 2) * 16; c < P.tn; c += 32) {
    uint32_t r[16];
    if (ok && nkb > 0) {
      tc_ld16_async(tmem + ((uint32_t)(32 * q) << 16) + c, r);
      tc_wait_ld();
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) r[e] = ok ? 0u : 0x7fc00000u;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (c + e < T) part[(c + e) * 128 + 32 * q + lane] = __uint_as_float(r[e]);
  }
  tc_fence_before();
  __syncwarp();
  if (splits > 1) cluster_sync();
  else __syncthreads();
  const Epilogue& E = P.e;
  for (int i = rank * FEW_THREADS + threadIdx.x; i < T * 32; i += splits * FEW_THREADS) {
    const int t = i >> 5, c = 4 * (i & 31), col = n0 + c;
    const uint32_t at = base + 4 * (uint32_t)(t * 128 + c);
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (splits > 1) {
      float4 u[FEW_SPLIT];
#pragma unroll
      for (int s = 0; s < FEW_SPLIT; ++s)
        if (s < splits) u[s] = ld_cluster(at, s);
#pragma unroll
      for (int s = 0; s < FEW_SPLIT; ++s)
        if (s < splits) v[0] += u[s].x, v[1] += u[s].y, v[2] += u[s].z, v[3] += u[s].w;
    } else {
      const float4 u = *(const float4*)(part + t * 128 + c);
      v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
    }
    const long row = t0 + t;
    const float xs = F8 ? E.x_scale[row] : 1.f;
    float z[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool on = col + e < P.N;
      const float s = F8 && on ? xs * E.w_scale[col + e] : 1.f;
      z[e] = fmaf(v[e], s, E.bias && on ? to_f32(E.bias[col + e]) : 0.f);
      v[e] = z[e];
    }
    activate(E.act, v);
    if (P.vec && col + 3 < P.N) {
      if (E.residual) {
        const uint2 r = *(const uint2*)(E.residual + row * E.ldr + col);
        const float2 a = bf2(r.x), b = bf2(r.y);
        v[0] += a.x, v[1] += a.y, v[2] += b.x, v[3] += b.y;
      }
      if (E.pre)
        *(uint2*)(E.pre + row * E.ldp + col) =
            make_uint2(to_bf2(make_float2(z[0], z[1])), to_bf2(make_float2(z[2], z[3])));
      *(uint2*)(E.y + row * E.ldy + col) = make_uint2(to_bf2(make_float2(v[0], v[1])), to_bf2(make_float2(v[2], v[3])));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < P.N) {
          if (E.residual) v[e] += to_f32(E.residual[row * E.ldr + col + e]);
          if (E.pre) E.pre[row * E.ldp + col + e] = __float2bfloat16_rn(z[e]);
          E.y[row * E.ldy + col + e] = __float2bfloat16_rn(v[e]);
        }
    }
  }
  __syncwarp();
  if (splits > 1) cluster_sync();  // a CTA's shared memory outlives its neighbours' reads
  else __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(P.cols) : "memory");
  }
}

// How a product of few tokens is cut: tokens and blocks of K of a CTA, CTAs of a cluster, and
// what it takes in ns, as measured.  Stages arrive at 110 bytes a ns an SM; two CTAs share one up
// to 128 tokens (108 KiB each; with 128 columns of TMEM at most, so that neither waits for the
// other's), above there is one.  A launch takes 3.1 us, with a cluster 4.8, and a tile's way out through
// shared memory 30 ns a token, 60 where one CTA does it alone.  More than eight clusters of eight CTAs that
// fill an SM wait for eight free SMs of a GPC (256 tokens of 2048 x 2048: 20.2 us with eight, 14 with four).
struct FewPlan {
  int tn, nt, tb, splits, per;
  long ns;
};
FewPlan few_plan(long T, long N, long nkb) {
  FewPlan best = {};
  const long tb = (T + FEW_T - 1) / FEW_T, nt = (N + 127) / 128, tn = ((T + tb - 1) / tb + 15) / 16 * 16;
  if (nt > 65535 || tb > 65535) return best;  // (a grid's limits: never few)
  const long per_sm = tn <= 128 ? 2 : 1;
  const int most = per_sm == 2 || nt * tb <= 8 ? FEW_SPLIT : FEW_SPLIT / 2;
  for (int s = 1; s <= most && (s == 1 || nkb >= 4 * s); s *= 2) {
    const long ctas = nt * tb * s, per = (nkb + s - 1) / s, waves = (ctas + SMS * per_sm - 1) / (SMS * per_sm);
    const long sharing = std::min(per_sm, (ctas + SMS - 1) / SMS);
    const long ns = (s > 1 ? 4800 + waves * 30 * tn : 3100 + waves * 60 * tn) +
                    waves * (per * sharing * (A_BYTES + tn * KB) / 110);
    if (s == 1 || ns <= best.ns) best = {(int)tn, (int)nt, (int)tb, s, (int)per, ns};
  }
  return best;
}
// What tiles of 256 x 256 by pairs of SMs take, in ns; 3 us more a round where rows of N side by side
// cannot leave by TMA.  (Rows that lie otherwise do not count: the form, and with it the order of the
// sums, goes by the sizes and the type, not by where the output is.)
long pairs_ns(long T, long N, long nkb) {
  const long tiles = ((T + BM - 1) / BM) * ((N + BN - 1) / BN);
  return 4500 + (tiles + SMS / 2 - 1) / (SMS / 2) * (nkb * 290 + (N % 8 == 0 ? 0 : 3000));
}

template <bool F8>
lx_status launch_few(Few& P, const FewPlan& L, int es, const lx_linear_desc* d, cudaStream_t st) {
  static bool cap[64] = {};
  int dev = 0;
  LX_CUDA(cudaGetDevice(&dev));
  LX_CUDA(smem_cap_once((const void*)k_linear_few<F8>, 224 * 1024, dev, cap));
  P.tn = L.tn;
  P.per = L.per;
  if (!encode_bytes_2d(&P.w, d->w, (long)d->K * es, d->N, d->ldw * es, 128) ||
      !encode_bytes_2d(&P.x, d->x, (long)d->K * es, d->T, d->ldx * es, P.tn))
    return fail(LX_ERR_CUDA, "cuTensorMapEncodeTiled(linear) failed");
  const int stage = A_BYTES + P.tn * KB, budget = P.tn <= 128 ? 108 * 1024 : 200 * 1024;
  P.cols = 32;
  while (P.cols < P.tn) P.cols *= 2;
  P.stages = std::min(16, budget / stage);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(L.splits, L.nt, L.tb);
  cfg.blockDim = dim3(FEW_THREADS);
  cfg.dynamicSmemBytes = budget + 1024;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = L.splits;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  LX_CUDA(cudaLaunchKernelEx(&cfg, k_linear_few<F8>, P));
  return LX_OK;
}

// ---------------------------------------------------------------------------
// the gradient of z, and the sums of its columns
// ---------------------------------------------------------------------------
struct DzArgs {
  int T, N, act, chunk;  // rows of a CTA
  const __nv_bfloat16 *dy, *pre;
  long lddy, ldp;
  __nv_bfloat16* dz;     // or NULL
  long ldz;
  float* part;           // [CTAs of rows][N], or NULL
};

// d times the activation's derivative, in pairs (gelu: see gelu2)
template <int ACT>
__device__ __forceinline__ float2 through(float2 d, float2 z) {
  const float2 one = both(1.f);
  if (ACT == RELU) return make_float2(z.x > 0.f ? d.x : d.x * 0.f, z.y > 0.f ? d.y : d.y * 0.f);
  if (ACT == SILU) {
    const float2 a = mul2(z, both(-LOG2E));
    const float2 q = add2(make_float2(ex2(a.x), ex2(a.y)), one);
    const float2 s = make_float2(rcp(q.x), rcp(q.y));
    return mul2(d, mul2(s, fma2(z, fma2(s, both(-1.f), one), one)));
  }
  if (ACT == GELU) {
    const float2 a = make_float2(fminf(fabsf(z.x), 100.f), fminf(fabsf(z.y), 100.f));
    const float2 q = fma2(a, both(0.3275911f * 0.70710678f), one);
    const float2 t = make_float2(rcp(q.x), rcp(q.y));
    const float2 s = mul2(mul2(a, a), both(-0.5f * LOG2E));
    const float2 e = make_float2(ex2(s.x), ex2(s.y));
    float2 p = fma2(both(-0.5f * 1.061405429f), t, both(0.5f * 1.453152027f));
    p = fma2(p, t, both(-0.5f * 1.421413741f));
    p = fma2(p, t, both(0.5f * 0.284496736f));
    p = fma2(p, t, both(-0.5f * 0.254829592f));
    p = fma2(mul2(p, t), e, both(0.5f));  // half the probability of (-|z|, |z|)
    const float2 cdf = add2(make_float2(copysignf(p.x, z.x), copysignf(p.y, z.y)), both(0.5f));
    return mul2(d, fma2(mul2(z, both(0.3989422804014327f)), e, cdf));
  }
  return d;
}

// dz is rounded to bf16 as the tensor cores take it (2^-9 of each term of the gradients' fp32
// sums); the bias's gradient sums it unrounded.  A warp reads rows of 32 VEC columns, AHEAD of them at
// a time.
template <int VEC, int ACT>
__global__ void __launch_bounds__(256, 4) k_linear_dz(const __grid_constant__ DzArgs A) {
  pdl_wait();
  __shared__ float sums[8][32 * VEC];
  constexpr int W = VEC == 8 ? 4 : 1, AHEAD = 4;  // words of a piece; rows
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int col = (blockIdx.x * 32 + lane) * VEC;
  const long t0 = (long)blockIdx.y * A.chunk;
  const int n = (int)min((long)A.chunk, A.T - t0);
  float s[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[e] = 0.f;
  auto read = [&](const __nv_bfloat16* p, uint32_t (&w)[W]) {
    if constexpr (VEC == 8) {
      const uint4 v = *(const uint4*)p;
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {
      w[0] = *(const uint16_t*)p;
    }
  };
  if (col < A.N) {
    for (int r0 = warp; r0 < n; r0 += 8 * AHEAD) {
      uint32_t a[AHEAD][W], b[AHEAD][W];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (r0 + 8 * i < n) {
          const long t = t0 + r0 + 8 * i;
          read(A.dy + t * A.lddy + col, a[i]);
          if (ACT != NONE) read(A.pre + t * A.ldp + col, b[i]);
        }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (r0 + 8 * i < n) {
          float d[VEC];
#pragma unroll
          for (int e = 0; e < VEC; e += 2) {
            const float2 v = through<ACT>(bf2(a[i][e / 2]), ACT != NONE ? bf2(b[i][e / 2]) : make_float2(0.f, 0.f));
            d[e] = v.x;
            if constexpr (VEC > 1) d[e + 1] = v.y;
          }
#pragma unroll
          for (int e = 0; e < VEC; ++e) s[e] += d[e];
          if (A.dz) store<__nv_bfloat16, VEC>(A.dz + (t0 + r0 + 8 * i) * A.ldz + col, d);
        }
    }
  }
  if (!A.part) return;
#pragma unroll
  for (int e = 0; e < VEC; ++e) sums[warp][lane * VEC + e] = s[e];
  __syncthreads();
  for (int c = threadIdx.x; c < 32 * VEC; c += 256) {
    const int at = blockIdx.x * 32 * VEC + c;
    if (at >= A.N) break;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += sums[w][c];
    A.part[(long)blockIdx.y * A.N + at] = v;
  }
}

template <int VEC>
void launch_dz(const DzArgs& A, dim3 grid, cudaStream_t st) {
  if (A.act == RELU) k_linear_dz<VEC, RELU><<<grid, 256, 0, st>>>(A);
  else if (A.act == SILU) k_linear_dz<VEC, SILU><<<grid, 256, 0, st>>>(A);
  else if (A.act == GELU) k_linear_dz<VEC, GELU><<<grid, 256, 0, st>>>(A);
  else k_linear_dz<VEC, NONE><<<grid, 256, 0, st>>>(A);
}

// the bias's gradient by itself (otherwise it is added up beside the products)
__global__ void __launch_bounds__(64) k_linear_db(const float* part, int chunks, int N, __nv_bfloat16* db) {
  pdl_wait();
  const int c = blockIdx.x * 64 + threadIdx.x;
  if (c < N) db[c] = __float2bfloat16_rn(column_sum(part, chunks, N, c));
}

// rows of a CTA of k_linear_dz: about four CTAs an SM; a multiple of the warps.  (All of few rows in one
// CTA, which would save the parts: 257 rows of 1003 14 us instead of 5.)
int dz_chunk(int T, int N) {
  const long cols = (N + 255) / 256;
  const long ctas = std::max(1L, 4L * SMS / cols);
  return (int)std::max(8L, std::min<long>(1L << 20, (((long)T + ctas - 1) / ctas + 7) / 8 * 8));
}
int dz_chunks(int T, int N) { return (int)(((long)T + dz_chunk(T, N) - 1) / dz_chunk(T, N)); }
size_t al(size_t v) { return (v + 255) / 256 * 256; }
// ranges of K of a product of M x N outputs: few tiles of long sums are cut, so that every pair of
// SMs has one, into ranges of 2048 at least
int grad_slices(long M, long N, long K) {
  const long tiles = ((M + BM - 1) / BM) * ((N + BN - 1) / BN);
  return (int)std::max(1L, std::min(std::min((long)MAX_SLICES, (long)(SMS / 2) / tiles), K / 2048));
}
size_t grad_blocks(long M, long N, long K) {
  const int s = grad_slices(M, N, K);
  return s > 1 ? al(4 * block_floats(M, N, s)) : 0;
}
long dz_ld(int N) { return ((long)N + 7) / 8 * 8; }

constexpr int MAX_T = 1 << 30, MAX_DIM = 1 << 24;

lx_status check_sizes(int32_t T, int32_t N, int32_t K, int32_t dtype) {
  if (T < 0) return fail(LX_ERR_ARG, "T < 0");
  if (T > MAX_T) return fail(LX_ERR_SHAPE, "T is above 2^30");
  if (N < 1 || N > MAX_DIM || K < 1 || K > MAX_DIM) return fail(LX_ERR_SHAPE, "N and K must be in 1..2^24");
  if (K % (dtype == LX_E4M3 ? 16 : 8) != 0) return fail(LX_ERR_SHAPE, "K must be a multiple of 16 bytes");
  // tiles of 256 x 256 are counted in 31 bits
  const long mt = ((long)T + 255) / 256, nt = ((long)N + 255) / 256, kt = ((long)K + 255) / 256;
  if (std::max(mt * nt, std::max(mt * kt, nt * kt)) > (1L << 30)) return fail(LX_ERR_SHAPE, "too many tiles");
  return LX_OK;
}

lx_status check_desc(const lx_linear_desc* d) {
  if (!d) return fail(LX_ERR_ARG, "desc is NULL");
  if (d->dtype != LX_BF16 && d->dtype != LX_E4M3) return fail(LX_ERR_ARG, "dtype must be LX_BF16 or LX_E4M3");
  if (d->act < LX_ACT_NONE || d->act > LX_ACT_GELU) return fail(LX_ERR_ARG, "unknown activation");
  LX_TRY(check_sizes(d->T, d->N, d->K, d->dtype));
  const int64_t per = d->dtype == LX_E4M3 ? 16 : 8;
  if (d->ldw < d->K || d->ldw % per != 0 || d->ldw > MAX_DIM) return fail(LX_ERR_SHAPE, "ldw");
  if (d->ldx < d->K || d->ldx % per != 0 || d->ldx > MAX_DIM) return fail(LX_ERR_SHAPE, "ldx");
  if (!d->w || !aligned(d->w, 16)) return fail(LX_ERR_ARG, "w is NULL or not 16-byte aligned");
  if (d->T > 0 && (!d->x || !aligned(d->x, 16))) return fail(LX_ERR_ARG, "x is NULL or not 16-byte aligned");
  return LX_OK;
}

}  // namespace
}  // namespace lx

extern "C" lx_status lx_linear(const lx_linear_desc* d, void* y, int64_t ldy, void* pre, void* stream) {
  using namespace lx;
  LX_TRY(check_desc(d));
  const bool f8 = d->dtype == LX_E4M3;
  const int es = f8 ? 1 : 2;
  if (f8 != (d->x_scale != nullptr) || f8 != (d->w_scale != nullptr))
    return fail(LX_ERR_ARG, "x_scale and w_scale go with LX_E4M3");
  if (!aligned(d->x_scale, 4) || !aligned(d->w_scale, 4) || !aligned(d->bias, 2) || !aligned(d->residual, 2) ||
      !aligned(y, 2) || !aligned(pre, 2))
    return fail(LX_ERR_ARG, "a pointer is not aligned to its element");
  if (d->T == 0) return LX_OK;
  if (!y) return fail(LX_ERR_ARG, "y is NULL");
  if (ldy < d->N || (d->residual && d->ldr < d->N)) return fail(LX_ERR_SHAPE, "rows are closer than N elements");
  if (ldy > (1L << 30) || (d->residual && d->ldr > (1L << 30))) return fail(LX_ERR_SHAPE, "rows are above 2^30 elements apart");
  const size_t sy = span(d->T, d->N, ldy, 2), sp = pre ? span(d->T, d->N, d->N, 2) : 0;
  const size_t sx = span(d->T, d->K, d->ldx, es), sw = span(d->N, d->K, d->ldw, es);
  const size_t sr = d->residual ? span(d->T, d->N, d->ldr, 2) : 0;
  const bool in_place = y == d->residual && d->ldr == ldy;
  const void* ins[] = {d->x, d->w, d->x_scale, d->w_scale, d->bias};
  const size_t sizes[] = {sx, sw, 4 * (size_t)d->T, 4 * (size_t)d->N, 2 * (size_t)d->N};
  for (int i = 0; i < 5; ++i)
    if (overlap(y, sy, ins[i], sizes[i]) || overlap(pre, sp, ins[i], sizes[i]))
      return fail(LX_ERR_ARG, "an output overlaps an input");
  if ((!in_place && overlap(y, sy, d->residual, sr)) || overlap(pre, sp, d->residual, sr))
    return fail(LX_ERR_ARG, "an output overlaps an input");
  if (overlap(y, sy, pre, sp)) return fail(LX_ERR_ARG, "two outputs overlap");

  const CallWaits waits = take_call_waits();
  Launch P = {};
  P.wait_cycles = waits.cycles;
  P.unmet = waits.unmet == LX_WAIT_CALL_PRODUCT;
  P.x_scale = d->x_scale;
  P.w_scale = d->w_scale;
  P.bias = (const __nv_bfloat16*)d->bias;
  P.residual = (const __nv_bfloat16*)d->residual;
  P.y = (__nv_bfloat16*)y;
  P.pre = (__nv_bfloat16*)pre;
  P.ldr = d->ldr;
  P.ldy = ldy;
  P.ldp = d->N;
  P.act = d->act;
  auto wide = [](const void* p, long ld, int b) { return !p || (((uintptr_t)p | (uintptr_t)(2 * ld)) % b) == 0; };
  cudaStream_t st = (cudaStream_t)stream;
  // Few tokens or tiles, by what the two forms take (µs, 2048 x 2048: 128 tokens 10.0 and 14.2, 1024 18.4
  // and 14.4; 512 x 8192 inputs: 21.8 and 40.8; 256 x 512 inputs: 13.8 and 7.5)
  const long nkb = ((long)d->K * es + KB - 1) / KB;
  const FewPlan few = few_plan(d->T, d->N, nkb);
  if (few.splits && few.ns < pairs_ns(d->T, d->N, nkb)) {
    Few F = {};
    F.e = P;
    F.T = d->T;
    F.N = d->N;
    F.nkb = (int)nkb;
    F.vec = wide(y, ldy, 8) && wide(pre, d->N, 8) && wide(d->residual, d->ldr, 8);
    return f8 ? launch_few<true>(F, few, es, d, st) : launch_few<false>(F, few, es, d, st);
  }
  P.tma_y = boxes(&P.map_y, y, d->N, d->T, ldy);
  P.tma_p = pre && boxes(&P.map_p, pre, d->N, d->T, d->N);
  P.tma_r = d->residual && boxes(&P.map_r, d->residual, d->N, d->T, d->ldr);
  P.n = 1;
  Problem& p = P.p[0];
  p.M = d->T;
  p.N = d->N;
  p.K = d->K;
  p.slices = 1;
  if (!operand(&p.a, d->x, d->K, d->T, d->ldx, es, false) || !operand(&p.b, d->w, d->K, d->N, d->ldw, es, false))
    return fail(LX_ERR_CUDA, "cuTensorMapEncodeTiled(linear) failed");
  return f8 ? launch_product<LINEAR, true>(P, st) : launch_product<LINEAR, false>(P, st);
}

extern "C" lx_status lx_linear_workspace(int32_t T, int32_t N, int32_t K, uint64_t* bytes) {
  using namespace lx;
  if (!bytes) return fail(LX_ERR_ARG, "bytes is NULL");
  LX_TRY(check_sizes(T, N, K, LX_BF16));
  *bytes = T == 0 ? 0
                  : al(2 * (size_t)T * dz_ld(N)) + al(4 * (size_t)dz_chunks(T, N) * N) + grad_blocks(T, K, N) +
                        grad_blocks(N, K, T);
  return LX_OK;
}

extern "C" lx_status lx_linear_backward(const lx_linear_desc* d, const void* dy, int64_t lddy, const void* pre,
                                        void* dx, void* dw, void* dbias, void* workspace, uint64_t workspace_bytes,
                                        void* stream) {
  using namespace lx;
  LX_TRY(check_desc(d));
  if (d->dtype != LX_BF16) return fail(LX_ERR_UNSUPPORTED, "the gradients are those of the bf16 product");
  if (!aligned(dx, 16) || !aligned(dw, 16)) return fail(LX_ERR_ARG, "dx and dw must be 16-byte aligned");
  if (!aligned(dy, 2) || !aligned(pre, 2) || !aligned(dbias, 2))
    return fail(LX_ERR_ARG, "a pointer is not aligned to its element");
  if (!dx && !dw && !dbias) return fail(LX_ERR_ARG, "no gradient is asked for");
  const int T = d->T, N = d->N, K = d->K;
  cudaStream_t st = (cudaStream_t)stream;
  if (T == 0) {
    if (dw) LX_CUDA(cudaMemsetAsync(dw, 0, 2 * (size_t)N * K, st));
    if (dbias) LX_CUDA(cudaMemsetAsync(dbias, 0, 2 * (size_t)N, st));
    return LX_OK;
  }
  if (!dy) return fail(LX_ERR_ARG, "dy is NULL");
  if ((d->act != LX_ACT_NONE) != (pre != nullptr)) return fail(LX_ERR_ARG, "pre goes with an activation");
  if (lddy < N) return fail(LX_ERR_SHAPE, "rows are closer than N elements");
  if (lddy > (1L << 30)) return fail(LX_ERR_SHAPE, "rows are above 2^30 elements apart");
  uint64_t need = 0;
  LX_TRY(lx_linear_workspace(T, N, K, &need));
  if (!workspace || !aligned(workspace, 256)) return fail(LX_ERR_ARG, "workspace is NULL or not 256-byte aligned");
  if (workspace_bytes < need) return fail(LX_ERR_ARG, "workspace too small");
  const void* ins[] = {d->x, d->w, dy, pre};
  const size_t in_n[] = {span(T, K, d->ldx, 2), span(N, K, d->ldw, 2), span(T, N, lddy, 2), pre ? 2 * (size_t)T * N : 0};
  const void* outs[] = {dx, dw, dbias, workspace};
  const size_t out_n[] = {2 * (size_t)T * K, 2 * (size_t)N * K, 2 * (size_t)N, need};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 4; ++j)
      if (overlap(outs[i], out_n[i], ins[j], in_n[j])) return fail(LX_ERR_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], out_n[i], outs[j], out_n[j])) return fail(LX_ERR_ARG, "two outputs overlap");
  }
  const CallWaits waits = take_call_waits();
  // dy itself is dz where nothing changes it and TMA can read it
  const bool direct = d->act == LX_ACT_NONE && aligned(dy, 16) && lddy % 8 == 0 && lddy <= MAX_DIM;
  __nv_bfloat16* dz = (__nv_bfloat16*)workspace;
  float* part = (float*)((char*)workspace + al(2 * (size_t)T * dz_ld(N)));
  const int chunk = dz_chunk(T, N), chunks = dz_chunks(T, N);
  if (!direct || dbias) {
    DzArgs A = {T, N, d->act, chunk, (const __nv_bfloat16*)dy, (const __nv_bfloat16*)pre, (long)lddy, (long)N,
                direct ? nullptr : dz, dz_ld(N), dbias ? part : nullptr};
    const bool vec = N % 8 == 0 && lddy % 8 == 0 && aligned(dy, 16) && aligned(pre, 16);
    if (vec) launch_dz<8>(A, dim3((N + 255) / 256, chunks), st);
    else launch_dz<1>(A, dim3((N + 31) / 32, chunks), st);
    LX_CUDA(cudaGetLastError());
    if (dbias && !dx && !dw)
      LX_TRY(launch_after(k_linear_db, dim3((N + 63) / 64), dim3(64), 0, 1, st, (const float*)part, chunks, N,
                          (__nv_bfloat16*)dbias));
  }
  if (!dx && !dw) return LX_OK;
  const void* g = direct ? dy : dz;
  const long ldg = direct ? lddy : dz_ld(N);
  Launch P = {};
  P.wait_cycles = waits.cycles;
  P.unmet = waits.unmet == LX_WAIT_CALL_PRODUCT;
  if (dbias) {
    P.db = (__nv_bfloat16*)dbias;
    P.db_part = part;
    P.db_chunks = chunks;
    P.db_n = N;
  }
  bool ok = true;
  Join joins[2];
  int n_joins = 0;
  float* blocks = (float*)((char*)part + al(4 * (size_t)chunks * N));
  // out by TMA, or its ranges' sums into the workspace, to be joined
  auto target = [&](Problem& p, void* out) {
    p.slices = grad_slices(p.M, p.N, p.K);
    if (p.slices == 1) return boxes(&p.out, out, p.N, p.M, p.N);
    p.blocks = blocks;
    joins[n_joins++] = Join{blocks, p.M, p.N, p.slices, nullptr, nullptr, nullptr, (__nv_bfloat16*)out};
    blocks += grad_blocks(p.M, p.N, p.K) / 4;
    return true;
  };
  // the product with the longer sums first: the shorter tiles even out the SMs' ends
  for (int i = 0; i < 2; ++i) {
    if ((N >= T) == (i == 0)) {
      if (!dx) continue;
      Problem& p = P.p[P.n++];
      p.M = T, p.N = K, p.K = N;
      p.b_mn = 1;
      ok = ok && target(p, dx) && operand(&p.a, g, N, T, ldg, 2, false) && operand(&p.b, d->w, K, N, d->ldw, 2, true);
    } else {
      if (!dw) continue;
      Problem& p = P.p[P.n++];
      p.M = N, p.N = K, p.K = T;
      p.a_mn = p.b_mn = 1;
      ok = ok && target(p, dw) && operand(&p.a, g, N, T, ldg, 2, true) && operand(&p.b, d->x, K, T, d->ldx, 2, true);
    }
  }
  if (!ok) return fail(LX_ERR_CUDA, "cuTensorMapEncodeTiled(linear gradients) failed");
  LX_TRY((launch_product<GRAD, false>(P, st)));
  for (int i = 0; i < n_joins; ++i) LX_TRY(launch_join(joins[i], st));
  return LX_OK;
}
