// The router's balance loss with its per-expert counts (lx_router_balance) and its
// gradient with respect to the logits (lx_router_balance_backward).  Over the n
// tokens that count (mask not 0, some logit above -inf), with p = softmax(l):
//   c_e = tokens whose set of distinct valid ids holds e,   P_e = mean p_e,
//   balance = E sum_e c_e / (n k) P_e,   z = mean (log sum_e exp l_e)^2,
//   loss = alpha balance + beta z,
//   dl = dloss p (alpha E / (n^2 k) (c_e - sum_j c_j p_j) + 2 beta / n lse).
//
// Both are bound by reading the logits (and writing their gradient) once.  A token's
// row is held in the registers of 4 to 32 lanes (16 logits a lane, 32 above 512
// experts), so that a warp has several rows in flight and the shuffles of a row's
// maximum and sums serve all of them.  The column sums of p stay in registers over
// the rows of a lane and are added up per CTA, then over the CTAs by a second launch,
// each in a fixed order.
#include <algorithm>

#include "lx_rows.cuh"

namespace lx {
namespace {

using namespace rows;

constexpr int BAL_THREADS = 512;
constexpr int BAL_CTAS = 2 * 152;  // of the first launch at most

struct BalArgs {
  const void* logits;
  long ld;
  const int* ids;
  const uint8_t* mask;
  int T, E, k;
  float* lse;
  float* part_p;  // [CTAs][E + 1]: column sums of p, then the sum of lse^2
  int* part_c;    // [CTAs][E + 1]: counts, then the tokens that count
  // backward
  const int* counts;
  const float* dloss;
  float alpha, beta;
  void* dlogits;
};

template <int G>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int G>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// Row t's logits of this lane: pieces of VEC, piece c at expert (c * G + lane) * VEC;
// -inf outside
template <typename T, int VEC, int G, int EPL>
__device__ __forceinline__ void load_row(const BalArgs& A, long t, bool on, int lane, float* v) {
#pragma unroll
  for (int c = 0; c < EPL / VEC; ++c) {
    const int e = (c * G + lane) * VEC;
#pragma unroll
    for (int j = 0; j < VEC; ++j) v[c * VEC + j] = -INFINITY;
    if (on && e < A.E) load<T, VEC>((const T*)A.logits + t * A.ld + e, v + c * VEC);
  }
}

// p = softmax in place, the row's log-sum-exp returned; all -inf: p = 0 and -inf
template <int G, int EPL>
__device__ __forceinline__ float softmax_row(float* v) {
  float m = -INFINITY, s = 0.f;
#pragma unroll
  for (int i = 0; i < EPL; ++i) m = fmaxf(m, v[i]);  // a NaN shows in the sum
  m = lanes_max<G>(m);
  const float m0 = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    v[i] = __expf(v[i] - m0);
    s += v[i];
  }
  s = lanes_sum<G>(s);
  if (s == 0.f) return -INFINITY;
  const float inv = 1.f / s;
#pragma unroll
  for (int i = 0; i < EPL; ++i) v[i] *= inv;
  return m0 + logf(s);
}

template <typename T, int VEC, int G, int EPL>
__global__ void __launch_bounds__(BAL_THREADS)
k_balance_fwd(const BalArgs A) {
  constexpr int ROWS = BAL_THREADS / G;  // of the CTA at a time
  extern __shared__ float sm[];          // [E] counts (int), then [warps][E] column sums
  int* cnt = reinterpret_cast<int*>(sm);
  float* col = sm + A.E;
  __shared__ float zs[BAL_THREADS / 32];
  __shared__ int ns;
  const int lane = threadIdx.x % G, warp = threadIdx.x >> 5;
  for (int e = threadIdx.x; e < A.E; e += BAL_THREADS) cnt[e] = 0;
  if (threadIdx.x == 0) ns = 0;
  __syncthreads();
  float acc[EPL], z = 0.f;
  int n = 0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) acc[i] = 0.f;
  for (long t0 = (long)blockIdx.x * ROWS; t0 < A.T; t0 += (long)gridDim.x * ROWS) {
    const long t = t0 + threadIdx.x / G;
    const bool on = t < A.T && (!A.mask || A.mask[t]);
    float v[EPL];
    load_row<T, VEC, G, EPL>(A, t, on, lane, v);
    const float lse = softmax_row<G, EPL>(v);
    if (t < A.T && lane == 0) A.lse[t] = lse;
    if (lse == -INFINITY) continue;
#pragma unroll
    for (int i = 0; i < EPL; ++i) acc[i] += v[i];
    if (lane == 0) {
      z = fmaf(lse, lse, z);
      ++n;
    }
    const int* id = A.ids + t * A.k;
    for (int s = lane; s < A.k; s += G) {
      const int e = id[s];
      bool first = e >= 0 && e < A.E;
      for (int j = 0; j < s; ++j) first &= id[j] != e;
      if (first) atomicAdd(&cnt[e], 1);
    }
  }
  __syncwarp();
  // the rows of a warp, then the warps
#pragma unroll
  for (int i = 0; i < EPL; ++i)
#pragma unroll
    for (int o = G; o < 32; o <<= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
  z = warp_sum(z);
  if (n) atomicAdd(&ns, n);
  if ((threadIdx.x & 31) == 0) zs[warp] = z;
  if ((threadIdx.x & 31) < G)
#pragma unroll
    for (int c = 0; c < EPL / VEC; ++c)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int e = (c * G + lane) * VEC + j;
        if (e < A.E) col[(long)warp * A.E + e] = acc[c * VEC + j];
      }
  __syncthreads();
  float* pp = A.part_p + (long)blockIdx.x * (A.E + 1);
  int* pc = A.part_c + (long)blockIdx.x * (A.E + 1);
  for (int e = threadIdx.x; e < A.E; e += BAL_THREADS) {
    float s = 0.f;
    for (int w = 0; w < BAL_THREADS / 32; ++w) s += col[(long)w * A.E + e];
    pp[e] = s;
    pc[e] = cnt[e];
  }
  if (threadIdx.x == 0) {
    float s = 0.f;
    for (int w = 0; w < BAL_THREADS / 32; ++w) s += zs[w];
    pp[A.E] = s;
    pc[A.E] = ns;
  }
}

// Adds the CTAs' partial sums and forms the loss: one CTA, a thread to an expert
__global__ void __launch_bounds__(1024)
k_balance_sum(const float* __restrict__ part_p, const int* __restrict__ part_c, int parts, int E, int k, float alpha,
              float beta, int* counts, float* prob, float* loss) {
  __shared__ float buf[2][32];
  __shared__ int nsh;
  __shared__ float zsh;
  int turn = 0;
  const int e = threadIdx.x;
  float p = 0.f;
  int c = 0;
  if (e < E)
    for (int i = 0; i < parts; ++i) {
      p += part_p[(long)i * (E + 1) + e];
      c += part_c[(long)i * (E + 1) + e];
    }
  if (e == 0) {
    int n = 0;
    float z = 0.f;
    for (int i = 0; i < parts; ++i) {
      n += part_c[(long)i * (E + 1) + E];
      z += part_p[(long)i * (E + 1) + E];
    }
    nsh = n;
    zsh = z;
  }
  __syncthreads();
  const int n = nsh;
  const float inv = n ? 1.f / (float)n : 0.f;
  p *= inv;
  const float bal = group_sum<false>((float)c * p, buf, turn) * ((float)E * inv / (float)k);
  if (e < E) {
    counts[e] = c;
    prob[e] = p;
  }
  if (e == 0) {
    const float z = zsh * inv;
    counts[E] = n;
    loss[0] = alpha * bal + beta * z;
    loss[1] = bal;
    loss[2] = z;
  }
}

template <typename T, int VEC, int G, int EPL>
__global__ void __launch_bounds__(BAL_THREADS)
k_balance_bwd(const BalArgs A) {
  constexpr int ROWS = BAL_THREADS / G;
  const int lane = threadIdx.x % G;
  const float n = (float)A.counts[A.E], g = A.dloss ? *A.dloss : 1.f;
  const float a = n > 0.f ? g * A.alpha * (float)A.E / (n * n * (float)A.k) : 0.f;
  const float b = n > 0.f ? g * 2.f * A.beta / n : 0.f;
  float cnt[EPL];
#pragma unroll
  for (int c = 0; c < EPL / VEC; ++c)
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int e = (c * G + lane) * VEC + j;
      cnt[c * VEC + j] = e < A.E ? (float)A.counts[e] : 0.f;
    }
  for (long t0 = (long)blockIdx.x * ROWS; t0 < A.T; t0 += (long)gridDim.x * ROWS) {
    const long t = t0 + threadIdx.x / G;
    const float lse = t < A.T ? A.lse[t] : -INFINITY;
    float v[EPL];
    load_row<T, VEC, G, EPL>(A, t, lse != -INFINITY, lane, v);
    softmax_row<G, EPL>(v);
    float d = 0.f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) d = fmaf(cnt[i], v[i], d);
    d = lanes_sum<G>(d);
    if (t >= A.T) continue;
    const float zl = lse == -INFINITY ? 0.f : b * lse;
#pragma unroll
    for (int c = 0; c < EPL / VEC; ++c) {
      const int e = (c * G + lane) * VEC;
      if (e < A.E) {
        float o[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) o[j] = v[c * VEC + j] * fmaf(a, cnt[c * VEC + j] - d, zl);
        store<T, VEC>((T*)A.dlogits + t * A.E + e, o);
      }
    }
  }
}

size_t fwd_smem(int E) { return sizeof(float) * (size_t)E * (1 + BAL_THREADS / 32); }

// Lanes to a row: 16 logits a lane, 32 above 512 experts
template <typename T, int VEC, bool BWD>
lx_status launch_bal(const BalArgs& A, int grid, size_t smem, cudaStream_t s) {
  static bool cap_done[64] = {};
  if (!BWD && A.E > 512) {
    int dev = 0;
    LX_CUDA(cudaGetDevice(&dev));
    LX_CUDA(smem_cap_once((const void*)k_balance_fwd<T, VEC, 32, 32>, (int)fwd_smem(LX_MAX_EXPERTS), dev, cap_done));
  }
#define LX_BAL_CASE(G, EPL)                                                     \
  {                                                                             \
    if (BWD) k_balance_bwd<T, VEC, G, EPL><<<grid, BAL_THREADS, 0, s>>>(A);     \
    else k_balance_fwd<T, VEC, G, EPL><<<grid, BAL_THREADS, smem, s>>>(A);      \
  }
  if (A.E <= 64) LX_BAL_CASE(4, 16)
  else if (A.E <= 128) LX_BAL_CASE(8, 16)
  else if (A.E <= 256) LX_BAL_CASE(16, 16)
  else if (A.E <= 512) LX_BAL_CASE(32, 16)
  else LX_BAL_CASE(32, 32)
#undef LX_BAL_CASE
  LX_CUDA(cudaGetLastError());
  return LX_OK;
}

template <bool BWD>
lx_status launch_any(int dtype, bool vec, const BalArgs& A, int grid, size_t smem, cudaStream_t s) {
  if (dtype == LX_BF16)
    return vec ? launch_bal<__nv_bfloat16, 8, BWD>(A, grid, smem, s)
               : launch_bal<__nv_bfloat16, 1, BWD>(A, grid, smem, s);
  return vec ? launch_bal<float, 4, BWD>(A, grid, smem, s) : launch_bal<float, 1, BWD>(A, grid, smem, s);
}

int lanes_of(int E) { return E <= 64 ? 4 : E <= 128 ? 8 : E <= 256 ? 16 : 32; }

// CTAs of the first launch: a row for every lane group, a resident grid at most
int ctas_of(int T, int E) {
  const long rows = BAL_THREADS / lanes_of(E);
  return (int)std::min((long)BAL_CTAS, std::max(1L, ((long)T + rows - 1) / rows));
}

lx_status check(int dtype, int T, int E, int k) {
  if (dtype != LX_F32 && dtype != LX_BF16) return fail(LX_ERR_ARG, "unknown dtype");
  if (T < 0) return fail(LX_ERR_ARG, "T < 0");
  if (E < 1 || E > LX_MAX_EXPERTS) return fail(LX_ERR_ARG, "E must be in 1..LX_MAX_EXPERTS");
  if (k < 1 || k > LX_MAX_K) return fail(LX_ERR_ARG, "k must be in 1..LX_MAX_K");
  return LX_OK;
}

uint64_t ws_bytes(int T, int E) { return (uint64_t)ctas_of(T, E) * (E + 1) * 8; }

}  // namespace
}  // namespace lx

extern "C" lx_status lx_router_balance_workspace(int32_t T, int32_t E, uint64_t* bytes) {
  using namespace lx;
  LX_TRY(check(LX_F32, T, E, 1));
  if (!bytes) return fail(LX_ERR_ARG, "bytes is NULL");
  *bytes = ws_bytes(T, E);
  return LX_OK;
}

extern "C" lx_status lx_router_balance(int32_t dtype, const void* logits, int64_t ld, const int32_t* topk_id,
                                       const uint8_t* mask, int32_t T, int32_t E, int32_t k, float balance_coef,
                                       float z_coef, int32_t* counts, float* prob, float* lse, float* loss,
                                       void* workspace, uint64_t workspace_bytes, void* stream) {
  using namespace lx;
  LX_TRY(check(dtype, T, E, k));
  const size_t es = dtype == LX_BF16 ? 2 : 4;
  if (!counts || !prob || !loss) return fail(LX_ERR_ARG, "counts, prob or loss is NULL");
  if (!workspace || !aligned(workspace, 16)) return fail(LX_ERR_ARG, "workspace is NULL or not 16-byte aligned");
  if (workspace_bytes < ws_bytes(T, E)) return fail(LX_ERR_ARG, "workspace too small");
  if (T > 0) {
    if (!logits || !topk_id || !lse) return fail(LX_ERR_ARG, "logits, topk_id or lse is NULL");
    if (ld < E) return fail(LX_ERR_SHAPE, "rows are closer than E elements");
  }
  if (!aligned(logits, es) || !aligned(topk_id, 4) || !aligned(counts, 4) || !aligned(prob, 4) || !aligned(lse, 4) ||
      !aligned(loss, 4))
    return fail(LX_ERR_ARG, "a pointer is not aligned to its element");
  cudaStream_t s = (cudaStream_t)stream;
  const int grid = ctas_of(T, E);
  BalArgs A = {};
  A.logits = logits;
  A.ld = ld;
  A.ids = topk_id;
  A.mask = mask;
  A.T = T;
  A.E = E;
  A.k = k;
  A.lse = lse;
  A.part_p = (float*)workspace;
  A.part_c = (int*)workspace + (size_t)grid * (E + 1);
  const bool vec = E % (16 / es) == 0 && aligned(logits, 16) && ld * es % 16 == 0;
  LX_TRY(launch_any<false>(dtype, vec, A, grid, fwd_smem(E), s));
  k_balance_sum<<<1, (E + 31) / 32 * 32, 0, s>>>(A.part_p, A.part_c, grid, E, k, balance_coef, z_coef, counts, prob,
                                                 loss);
  LX_CUDA(cudaGetLastError());
  return LX_OK;
}

extern "C" lx_status lx_router_balance_backward(int32_t dtype, const void* logits, int64_t ld, const float* lse,
                                                const int32_t* counts, const float* dloss, int32_t T, int32_t E,
                                                int32_t k, float balance_coef, float z_coef, void* dlogits,
                                                void* stream) {
  using namespace lx;
  LX_TRY(check(dtype, T, E, k));
  if (T == 0) return LX_OK;
  const size_t es = dtype == LX_BF16 ? 2 : 4;
  if (!logits || !lse || !counts || !dlogits) return fail(LX_ERR_ARG, "logits, lse, counts or dlogits is NULL");
  if (ld < E) return fail(LX_ERR_SHAPE, "rows are closer than E elements");
  if (!aligned(logits, es) || !aligned(lse, 4) || !aligned(counts, 4) || !aligned(dloss, 4) || !aligned(dlogits, es))
    return fail(LX_ERR_ARG, "a pointer is not aligned to its element");
  if (!(dlogits == logits && ld == E) && overlap(dlogits, (size_t)T * E * es, logits, span(T, E, ld, es)))
    return fail(LX_ERR_ARG, "dlogits overlaps logits");
  BalArgs A = {};
  A.logits = logits;
  A.ld = ld;
  A.T = T;
  A.E = E;
  A.k = k;
  A.lse = const_cast<float*>(lse);
  A.counts = counts;
  A.dloss = dloss;
  A.alpha = balance_coef;
  A.beta = z_coef;
  A.dlogits = dlogits;
  const bool vec = E % (16 / es) == 0 && aligned(logits, 16) && ld * es % 16 == 0 && aligned(dlogits, 16);
  const long rows = BAL_THREADS / lanes_of(E);
  const int grid = (int)std::min(((long)T + rows - 1) / rows, 8L * 152);
  return launch_any<true>(dtype, vec, A, grid, 0, (cudaStream_t)stream);
}
