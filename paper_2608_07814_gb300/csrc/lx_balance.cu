// The router's balance loss with its per-expert counts (lx_router_balance) and its
// gradient with respect to the logits (lx_router_balance_backward).  Over the n
// tokens that count (mask not 0, some logit above -inf), with p = softmax(l):
//   c_e = tokens whose set of distinct valid ids holds e,   P_e = mean p_e,
//   balance = E sum_e c_e / (n k) P_e,   z = mean (log sum_e exp l_e)^2,
//   loss = alpha balance + beta z,
//   dl = dloss p (alpha E / (n^2 k) (c_e - sum_j c_j p_j) + 2 beta / n lse).
//
// Both are bound by reading the logits (and writing their gradient) once.  A token's
// row is held in the registers of 1 to 32 lanes (16 logits a lane; the forward 32 above 64
// experts, the backward above 512), so that a warp has several rows in flight and the shuffles of a row's
// maximum and sums serve all of them; the forward loads a lane's next row before it
// works on one.  The column sums of p stay in registers over the rows of a lane and are
// added up per CTA, then over the CTAs by a second launch that starts beside the first's
// last CTAs, each in a fixed order; one CTA finishes by itself.
#include <cooperative_groups.h>

#include <algorithm>

#include "lx_rows.cuh"

namespace lx {
namespace {

using namespace rows;

constexpr int BAL_THREADS = 256;
constexpr int BAL_WARPS = BAL_THREADS / 32;
constexpr int TILE = 256, TILE_WORDS = TILE / 32;  // tokens whose sets a CTA holds as bits
static_assert(TILE_WORDS == BAL_WARPS, "the warps' column sums take the bits' place");
constexpr int SUM_CTAS = 8, SUM_THREADS = 1024;  // the second launch: one cluster

struct BalArgs {
  const void* logits;
  long ld;
  const int* ids;
  const uint8_t* mask;
  int T, E, k;
  int chunk;  // tokens of a CTA of the forward
  float* lse;
  float* part_p;  // [CTAs][E + 1]: column sums of p, then the sum of lse^2
  int* part_c;    // [CTAs][E + 1]: counts, then the tokens that count
  int parts;      // CTAs of the first launch
  float alpha, beta;
  float *prob, *loss;
  int* counts;
  // backward
  const float* dloss;
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

// A lane's pieces of a row, as they are stored: VEC logits each, piece c at expert
// (c * G + lane) * VEC.  Pieces outside the row hold -inf from the start; a row that is
// not loaded leaves the previous one's values.
template <typename T, int VEC, int G, int EPL>
struct Raw {
  static constexpr int NCH = EPL / VEC;
  using P = typename std::conditional<VEC == 1, T, uint4>::type;
  P p[NCH];
  __device__ static int pieces(int E, int lane) {  // inside the row (they ascend)
    int n = 0;
#pragma unroll
    for (int c = 0; c < NCH; ++c) n += (c * G + lane) * VEC < E;
    return n;
  }
  __device__ void clear() {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if constexpr (VEC == 1) {
        p[c] = from_f32<T>(-INFINITY);
      } else {
        const uint32_t w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
        p[c] = make_uint4(w, w, w, w);
      }
    }
  }
  __device__ void load(const BalArgs& A, long t, int lane, int count) {
    const T* row = (const T*)A.logits + t * A.ld + lane * VEC;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
      if (c < count) p[c] = *(const P*)(row + c * G * VEC);
  }
  __device__ void get(float2* v) const {  // as pairs of fp32
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if constexpr (VEC == 1) {
        const float x = to_f32(p[c]);
        if (c & 1) v[c / 2].y = x;
        else v[c / 2].x = x;
      } else {
        const uint32_t w[4] = {p[c].x, p[c].y, p[c].z, p[c].w};
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j)
          v[c * (VEC / 2) + j] = sizeof(T) == 4
                                     ? make_float2(__uint_as_float(w[(2 * j) & 3]), __uint_as_float(w[(2 * j + 1) & 3]))
                                     : bf2(w[j & 3]);
      }
    }
  }
};

// v becomes exp(v - max); returns its sum's reciprocal, 0 for a row of nothing but -inf
// (a NaN shows in the sum), and the row's log-sum-exp
template <int G, int N2>
__device__ __forceinline__ float exp_row(float2* v, float& lse) {
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < N2; ++i) m = fmaxf(m, fmaxf(v[i].x, v[i].y));
  m = lanes_max<G>(m);
  const float m0 = m == -INFINITY ? 0.f : m;
  const float2 neg = both(-m0), l2e = both(1.4426950408889634f);
  float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
  for (int i = 0; i < N2; ++i) {
    v[i] = muls(adds(v[i], neg), l2e);
    v[i].x = ex2(v[i].x);
    v[i].y = ex2(v[i].y);
    s2 = adds(s2, v[i]);
  }
  const float s = lanes_sum<G>(s2.x + s2.y);
  lse = s == 0.f ? -INFINITY : m0 + logf(s);
  return s == 0.f ? 0.f : 1.f / s;
}

__device__ __forceinline__ void write_loss(const BalArgs& A, float bal, float z, int n) {
  const float inv = n ? 1.f / (float)n : 0.f;
  bal *= (float)A.E * inv / (float)A.k;
  z *= inv;
  A.counts[A.E] = n;
  A.loss[0] = A.alpha * bal + A.beta * z;
  A.loss[1] = bal;
  A.loss[2] = z;
}

template <typename T, int VEC, int G, int EPL>
__global__ void __launch_bounds__(BAL_THREADS, EPL == 16 ? 3 : 2)
k_balance_fwd(const __grid_constant__ BalArgs A) {
  constexpr int ROWS = BAL_THREADS / G, N2 = EPL / 2;  // ROWS: of the CTA at a time
  // [E] counts, then [TILE_WORDS][E] bits of the tile's sets, at the end [warps][E] sums
  extern __shared__ float sm[];
  int* cnt = reinterpret_cast<int*>(sm);
  uint32_t* bits = reinterpret_cast<uint32_t*>(sm) + A.E;
  float* col = sm + A.E;
  __shared__ float zs[BAL_WARPS], bs[BAL_WARPS];
  __shared__ int ns[BAL_WARPS];
  __shared__ uint32_t valid[TILE_WORDS];
  const int tid = threadIdx.x, lane = tid % G, warp = tid >> 5, wl = tid & 31;
  // this launch started after its predecessors had ended: the next may be scheduled
  if (A.parts > 1) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  float2 acc[N2];
  float z = 0.f;
  int n = 0;
#pragma unroll
  for (int i = 0; i < N2; ++i) acc[i] = make_float2(0.f, 0.f);
  Raw<T, VEC, G, EPL> raw;
  const int count = raw.pieces(A.E, lane);
  raw.clear();
  const long t_end = min((long)A.T, ((long)blockIdx.x + 1) * A.chunk);
  // a lane holds its row, and the next one is on its way (a masked one too: its values
  // are not used)
  auto masked_in = [&](long t) { return t < t_end && (!A.mask || A.mask[t]); };
  long t = (long)blockIdx.x * A.chunk + tid / G;
  bool on = masked_in(t);
  if (t < t_end) raw.load(A, t, lane, count);
  for (int e = tid; e < A.E; e += BAL_THREADS) cnt[e] = 0;
  for (long tile = (long)blockIdx.x * A.chunk; tile < t_end; tile += TILE) {
    const int rows = (int)min((long)TILE, t_end - tile), words = (rows + 31) / 32;
    for (int i = tid; i < words * A.E; i += BAL_THREADS) bits[i] = 0u;
    if (tid < TILE_WORDS) valid[tid] = 0u;
    __syncthreads();
    // a bit for every (token, expert) of the tile's sets: repeats fall together
    const int* ids = A.ids + tile * A.k;
    constexpr int U = 8;  // ids in flight a thread
    for (int q0 = tid; q0 < rows * A.k; q0 += U * BAL_THREADS) {
      int e[U];
#pragma unroll
      for (int u = 0; u < U; ++u) e[u] = q0 + u * BAL_THREADS < rows * A.k ? ids[q0 + u * BAL_THREADS] : -1;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (e[u] >= 0 && e[u] < A.E) {
          const int r = (q0 + u * BAL_THREADS) / A.k;
          atomicOr(&bits[(r >> 5) * A.E + e[u]], 1u << (r & 31));
        }
    }
    for (int r0 = 0; r0 < rows; r0 += ROWS) {
      float2 v[N2];
      raw.get(v);
      const bool now = on;
      const long row = t;
      t += ROWS;
      on = masked_in(t);
      if (t < t_end) raw.load(A, t, lane, count);
      float lse;
      const float inv = exp_row<G, N2>(v, lse);
      if (!now) lse = -INFINITY;
      if (row < t_end && lane == 0) A.lse[row] = lse;
      if (lse != -INFINITY) {
#pragma unroll
        for (int i = 0; i < N2; ++i) acc[i] = fmas(v[i], both(inv), acc[i]);
        if (lane == 0) {
          z = fmaf(lse, lse, z);
          ++n;
          const int r = (int)(row - tile);
          atomicOr(&valid[r >> 5], 1u << (r & 31));
        }
      }
      __syncwarp();
    }
    __syncthreads();
    for (int e = tid; e < A.E; e += BAL_THREADS) {
      int c = 0;
      for (int w = 0; w < words; ++w) c += __popc(bits[w * A.E + e] & valid[w]);
      cnt[e] += c;
    }
    __syncthreads();
  }
  // the rows of a warp, then the warps
#pragma unroll
  for (int i = 0; i < N2; ++i)
#pragma unroll
    for (int o = G; o < 32; o <<= 1) {
      acc[i].x += __shfl_xor_sync(0xffffffffu, acc[i].x, o);
      acc[i].y += __shfl_xor_sync(0xffffffffu, acc[i].y, o);
    }
  z = warp_sum(z);
  n = __reduce_add_sync(0xffffffffu, n);
  if (wl == 0) {
    zs[warp] = z;
    ns[warp] = n;
  }
  if (wl < G)
#pragma unroll
    for (int c = 0; c < EPL / VEC; ++c)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int e = (c * G + lane) * VEC + j, i = c * VEC + j;
        if (e < A.E) col[warp * A.E + e] = i & 1 ? acc[i / 2].y : acc[i / 2].x;
      }
  __syncthreads();
  z = 0.f;
  n = 0;
  for (int w = 0; w < BAL_WARPS; ++w) {
    z += zs[w];
    n += ns[w];
  }
  const bool alone = A.parts == 1;
  const float inv = n ? 1.f / (float)n : 0.f;
  float* pp = A.part_p + (long)blockIdx.x * (A.E + 1);
  int* pc = A.part_c + (long)blockIdx.x * (A.E + 1);
  float bal = 0.f;
  for (int e = tid; e < A.E; e += BAL_THREADS) {
    float s = 0.f;
    for (int w = 0; w < BAL_WARPS; ++w) s += col[w * A.E + e];
    if (alone) {
      A.counts[e] = cnt[e];
      A.prob[e] = s * inv;
      bal = fmaf((float)cnt[e], s * inv, bal);
    } else {
      pp[e] = s;
      pc[e] = cnt[e];
    }
  }
  if (!alone) {
    if (tid == 0) {
      pp[A.E] = z;
      pc[A.E] = n;
    }
    return;
  }
  bal = warp_sum(bal);
  if (wl == 0) bs[warp] = bal;
  __syncthreads();
  if (tid == 0) {
    bal = 0.f;
    for (int w = 0; w < BAL_WARPS; ++w) bal += bs[w];
    write_loss(A, bal, z, n);
  }
}

// Adds the CTAs' partial sums and forms the loss.  One cluster: CTA r takes the r-th 32
// of every 256 columns, 32 ranges of the parts each; every CTA adds up n and z for itself.
__global__ void __cluster_dims__(SUM_CTAS, 1, 1) __launch_bounds__(SUM_THREADS)
k_balance_sum(const __grid_constant__ BalArgs A) {
  __shared__ float sp[32][33], wz[32], wb[32], share[SUM_CTAS];
  __shared__ int sc[32][33], wn[32];
  cooperative_groups::cluster_group cl = cooperative_groups::this_cluster();
  cl.sync();  // all have started before one writes into another
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = (int)cl.block_rank(), E1 = A.E + 1;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float z = 0.f, bal = 0.f;
  int n = 0;
  for (int i = tid; i < A.parts; i += SUM_THREADS) {
    z += A.part_p[(long)i * E1 + A.E];
    n += A.part_c[(long)i * E1 + A.E];
  }
  z = warp_sum(z);
  n = __reduce_add_sync(0xffffffffu, n);
  if (lane == 0) {
    wz[warp] = z;
    wn[warp] = n;
  }
  __syncthreads();
  z = warp_sum(wz[lane]);
  n = __reduce_add_sync(0xffffffffu, wn[lane]);
  const float inv = n ? 1.f / (float)n : 0.f;
  for (int e0 = r * 32; e0 < A.E; e0 += SUM_CTAS * 32) {
    float p = 0.f;
    int q = 0;
    if (e0 + lane < A.E)
#pragma unroll 4
      for (int i = warp; i < A.parts; i += 32) {
        p += A.part_p[(long)i * E1 + e0 + lane];
        q += A.part_c[(long)i * E1 + e0 + lane];
      }
    sp[warp][lane] = p;
    sc[warp][lane] = q;
    __syncthreads();
    p = warp_sum(sp[lane][warp]);  // column e0 + warp
    q = __reduce_add_sync(0xffffffffu, sc[lane][warp]);
    if (lane == 0 && e0 + warp < A.E) {
      A.counts[e0 + warp] = q;
      A.prob[e0 + warp] = p * inv;
      bal += (float)q * (p * inv);
    }
    __syncthreads();
  }
  if (lane == 0) wb[warp] = bal;
  __syncthreads();
  if (warp == 0) {
    bal = warp_sum(wb[lane]);
    if (lane == 0) *cl.map_shared_rank(&share[r], 0) = bal;
  }
  cl.sync();
  if (r == 0 && tid == 0) {
    bal = 0.f;
    for (int i = 0; i < SUM_CTAS; ++i) bal += share[i];
    write_loss(A, bal, z, n);
  }
}

template <typename T, int VEC, int G, int EPL>
__global__ void __launch_bounds__(BAL_THREADS, EPL == 16 ? 4 : 2)
k_balance_bwd(const __grid_constant__ BalArgs A) {
  constexpr int ROWS = BAL_THREADS / G, N2 = EPL / 2;
  const int lane = threadIdx.x % G;
  const float n = (float)A.counts[A.E], g = A.dloss ? *A.dloss : 1.f;
  const float a = n > 0.f ? g * A.alpha * (float)A.E / (n * n * (float)A.k) : 0.f;
  const float b = n > 0.f ? g * 2.f * A.beta / n : 0.f;
  float2 cnt[N2];
#pragma unroll
  for (int c = 0; c < EPL / VEC; ++c)
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int e = (c * G + lane) * VEC + j, i = c * VEC + j;
      const float x = e < A.E ? (float)A.counts[e] : 0.f;
      if (i & 1) cnt[i / 2].y = x;
      else cnt[i / 2].x = x;
    }
  const int count = Raw<T, VEC, G, EPL>::pieces(A.E, lane);
  for (long t0 = (long)blockIdx.x * ROWS; t0 < A.T; t0 += (long)gridDim.x * ROWS) {
    const long t = t0 + threadIdx.x / G;
    const float lse = t < A.T ? A.lse[t] : -INFINITY;
    const bool on = lse != -INFINITY;
    Raw<T, VEC, G, EPL> raw;
    raw.clear();
    if (t < A.T) raw.load(A, t, lane, count);  // beside lse; a masked row's values are not used
    float2 v[N2];
    raw.get(v);
    float again;
    const float inv = exp_row<G, N2>(v, again);
    float2 d2 = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < N2; ++i) {
      v[i] = muls(v[i], both(inv));
      d2 = fmas(cnt[i], v[i], d2);
    }
    const float d = lanes_sum<G>(d2.x + d2.y);
    if (t >= A.T) continue;
    if (!on)
#pragma unroll
      for (int i = 0; i < N2; ++i) v[i] = make_float2(0.f, 0.f);
    const float2 base = both(on ? b * lse : 0.f), a2 = both(on ? a : 0.f), nd = both(on ? -d : 0.f);
    T* row = (T*)A.dlogits + t * A.E + lane * VEC;
#pragma unroll
    for (int c = 0; c < EPL / VEC; ++c) {
      if (c >= count) break;
      float o[VEC == 1 ? 2 : VEC];
      if constexpr (VEC == 1) {
        const float p = c & 1 ? v[c / 2].y : v[c / 2].x, q = c & 1 ? cnt[c / 2].y : cnt[c / 2].x;
        o[0] = p * fmaf(a2.x, q + nd.x, base.x);
      } else {
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) {
          const int i = c * (VEC / 2) + j;
          const float2 w = muls(v[i], fmas(a2, adds(cnt[i], nd), base));
          o[2 * j] = w.x;
          o[2 * j + 1] = w.y;
        }
      }
      store<T, VEC>(row + c * G * VEC, o);
    }
  }
}

size_t fwd_smem(int E) { return sizeof(float) * (size_t)E * (1 + TILE_WORDS); }
static_assert(LX_MAX_EXPERTS * 4 * (1 + BAL_WARPS) <= 47 * 1024, "no more shared memory than every launch may have");

// Lanes to a row
int lanes_of(int E, bool bwd) {
  int g = 1;
  while (g < 32 && g * (bwd || E <= 64 ? 16 : 32) < E) g *= 2;
  return g;
}

template <typename T, int VEC, bool BWD>
lx_status launch_bal(const BalArgs& A, int grid, size_t smem, cudaStream_t s) {
#define LX_BAL_CASE(G, EPL)                                                          \
  {                                                                                  \
    if constexpr (BWD) k_balance_bwd<T, VEC, G, EPL><<<grid, BAL_THREADS, 0, s>>>(A); \
    else k_balance_fwd<T, VEC, G, EPL><<<grid, BAL_THREADS, smem, s>>>(A);           \
  }
  const int lanes = lanes_of(A.E, BWD);
  if (A.E <= 16) LX_BAL_CASE(1, 16)
  else if (A.E <= 32) LX_BAL_CASE(2, 16)
  else if (A.E <= 64) LX_BAL_CASE(4, 16)
  else if (A.E > 512) LX_BAL_CASE(32, 32)
  else if constexpr (BWD) {
    if (lanes == 8) LX_BAL_CASE(8, 16)
    else if (lanes == 16) LX_BAL_CASE(16, 16)
    else LX_BAL_CASE(32, 16)
  } else {
    if (lanes == 4) LX_BAL_CASE(4, 32)
    else if (lanes == 8) LX_BAL_CASE(8, 32)
    else LX_BAL_CASE(16, 32)
  }
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

// Tokens of a CTA of the forward, in whole rounds of its rows, for a resident grid at most;
// up to two rounds one CTA does the whole call, which saves the second launch (E = 128: 64
// tokens 4.5 us against 5.8, 256 tokens 10.0 against 6.0)
int chunk_of(int T, int E) {
  const long rows = BAL_THREADS / lanes_of(E, false), ctas = SMS * (E <= 64 ? 3 : 2);
  if (T <= 2 * rows) return (int)(2 * rows);
  return (int)(((T + ctas - 1) / ctas + rows - 1) / rows * rows);
}
int ctas_of(int T, int E) { return std::max(1, (int)(((long)T + chunk_of(T, E) - 1) / chunk_of(T, E))); }

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
  A.chunk = chunk_of(T, E);
  A.parts = grid;
  A.alpha = balance_coef;
  A.beta = z_coef;
  A.prob = prob;
  A.loss = loss;
  A.counts = counts;
  const bool vec = E % (16 / es) == 0 && aligned(logits, 16) && ld * es % 16 == 0;
  LX_TRY(launch_any<false>(dtype, vec, A, grid, fwd_smem(E), s));
  if (grid == 1) return LX_OK;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(SUM_CTAS);
  cfg.blockDim = dim3(SUM_THREADS);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  LX_CUDA(cudaLaunchKernelEx(&cfg, k_balance_sum, A));
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
  A.counts = const_cast<int32_t*>(counts);
  A.dloss = dloss;
  A.alpha = balance_coef;
  A.beta = z_coef;
  A.dlogits = dlogits;
  const bool vec = E % (16 / es) == 0 && aligned(logits, 16) && ld * es % 16 == 0 && aligned(dlogits, 16);
  const long rows = BAL_THREADS / lanes_of(E, true);
  const int grid = (int)std::min(((long)T + rows - 1) / rows, 8L * SMS);
  return launch_any<true>(dtype, vec, A, grid, 0, (cudaStream_t)stream);
}
