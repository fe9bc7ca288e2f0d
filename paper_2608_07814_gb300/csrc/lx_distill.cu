// Distillation from a teacher's stored top logits (lx_distill_loss).  For a token
// with student logits z [V], teacher entries (id_j, t_j), weight w:
//   q_j = softmax_j(t_j / tau) over the valid entries, or exp(t_j / tau - L),
//   kd  = sum_j q_j (log q_j - log p_{id_j}),  p = softmax(z / tau),  m = sum_j q_j
//   ce  = log sum_v exp z_v - z_label
//   loss = w (a tau^2 kd + b ce)
//   dz_v = w (a tau (m p_v - sum_{j: id_j = v} q_j) + b (softmax(z)_v - [v = label])).
//
// Bound by the logits: one read of the row for its maximum and sums (kept per thread
// and joined once), a second one, which L2 serves, for the gradient that is written.
// The entries' places are written once more after the row, with what the dense part
// leaves out; entries of one id are added up.
#include <algorithm>

#include "lx_rows.cuh"

namespace lx {
namespace {

using namespace rows;

constexpr int DIS_THREADS = 512;
constexpr int DIS_WARPS = DIS_THREADS / 32;
constexpr int MAX_TEACHER = LX_MAX_TEACHER;

struct DistillArgs {
  const void* logits;
  long ld;
  const int* ids;
  const float* top;
  const float* top_lse;
  const int* labels;
  const float* weight;
  int T, V, K;
  float tau, a, b;
  float* loss;
  void* dlogits;
  long ldd;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Running maximum of a row part and its sums of exp((z - m) / tau) and exp(z - m);
// the maximum starts at the lowest finite value, so that a part of nothing but -inf
// has zero sums and no difference of infinities is formed
struct Run {
  float m = -3.402823466e38f, s = 0.f, s1 = 0.f;
};

template <bool TWO>
__device__ __forceinline__ void join(Run& r, float m, float s, float s1, float ct, float c1) {
  const float M = fmaxf(r.m, m);
  const float fr = ex2((r.m - M) * ct), fo = ex2((m - M) * ct);
  r.s = r.s * fr + s * fo;
  if (TWO) r.s1 = r.s1 * ex2((r.m - M) * c1) + s1 * ex2((m - M) * c1);
  r.m = M;
}

constexpr float LOG2E = 1.4426950408889634f;

// A row's vector part: from the first 16-byte boundary, in pieces of N elements
template <typename T>
struct Span {
  static constexpr int N = 16 / sizeof(T);
  int head, pieces;  // elements before it; pieces
  __device__ Span(const T* row, int V) {
    head = min(V, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T));
    pieces = (V - head) / N;
  }
};

// TWO: a hard-label term at another temperature than the teacher's
template <typename T, bool TWO>
__global__ void __launch_bounds__(DIS_THREADS)
k_distill(const DistillArgs A) {
  constexpr int N = Span<T>::N;
  __shared__ float rm[DIS_WARPS], rs[DIS_WARPS], rs1[DIS_WARPS];
  __shared__ int eid[MAX_TEACHER + 4];
  __shared__ float ez[MAX_TEACHER + 4], eq[MAX_TEACHER + 4], elq[MAX_TEACHER + 4];
  __shared__ float msum;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float ct = LOG2E / A.tau, c1 = LOG2E;
  for (long t = blockIdx.x; t < A.T; t += gridDim.x) {
    const T* z = (const T*)A.logits + t * A.ld;
    T* dz = A.dlogits ? (T*)A.dlogits + t * A.ldd : nullptr;
    const float w = A.weight ? A.weight[t] : 1.f;
    const Span<T> S(z, A.V);
    const bool same = dz && ((((uintptr_t)dz ^ (uintptr_t)z) & 15) == 0);
    Run r;
    const int label = A.labels ? A.labels[t] : -1;
    const bool hard = label >= 0 && label < A.V;
    if (w != 0.f) {
      if (warp == 0) {  // the teacher's entries; entry K is the label
        float tm = -INFINITY;
        for (int j = lane; j < A.K; j += 32) {
          const int id = A.ids[t * A.K + j];
          const bool ok = id >= 0 && id < A.V;
          const float v = ok ? A.top[t * A.K + j] : -INFINITY;
          eid[j] = ok ? id : -1;
          ez[j] = ok ? to_f32(z[id]) : 0.f;
          eq[j] = v;
          tm = fmaxf(tm, v);
        }
        if (lane == 0) {
          eid[A.K] = hard ? label : -1;
          ez[A.K] = hard ? to_f32(z[label]) : 0.f;
          eq[A.K] = 0.f;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) tm = fmaxf(tm, __shfl_xor_sync(0xffffffffu, tm, o));
        float lz;  // log of the distribution's sum, relative to tm / tau
        if (A.top_lse) {
          lz = A.top_lse[t] - tm / A.tau;
        } else {
          float s = 0.f;
          for (int j = lane; j < A.K; j += 32)
            if (eid[j] >= 0) s += tm == -INFINITY ? 0.f : expf((eq[j] - tm) / A.tau);
          lz = logf(warp_sum(s));
        }
        float m = 0.f;
        for (int j = lane; j < A.K; j += 32) {
          const float l = eid[j] >= 0 && eq[j] != -INFINITY ? (eq[j] - tm) / A.tau - lz : -INFINITY;
          const float q = expf(l);
          elq[j] = l;
          eq[j] = q;
          m += q;
        }
        m = warp_sum(m);
        if (lane == 0) msum = m;
      }
      auto take = [&](const float* v, int n) {
        float m = r.m;
        for (int j = 0; j < n; ++j) m = fmaxf(m, v[j]);
        if (m > r.m) {
          r.s *= ex2((r.m - m) * ct);
          if (TWO) r.s1 *= ex2((r.m - m) * c1);
          r.m = m;
        }
        for (int j = 0; j < n; ++j) {
          r.s += ex2((v[j] - r.m) * ct);
          if (TWO) r.s1 += ex2((v[j] - r.m) * c1);
        }
      };
      for (int p = tid; p < S.pieces; p += DIS_THREADS) {
        float v[N];
        load<T, N>(z + S.head + (long)p * N, v);
        take(v, N);
      }
      const int rest = A.V - S.head - S.pieces * N;
      if (tid < S.head + rest) {
        const float v = to_f32(z[tid < S.head ? tid : A.V - rest + tid - S.head]);
        take(&v, 1);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        join<TWO>(r, __shfl_xor_sync(0xffffffffu, r.m, o), __shfl_xor_sync(0xffffffffu, r.s, o),
                  TWO ? __shfl_xor_sync(0xffffffffu, r.s1, o) : 0.f, ct, c1);
      if (lane == 0) {
        rm[warp] = r.m;
        rs[warp] = r.s;
        rs1[warp] = r.s1;
      }
      __syncthreads();
      r = Run();
      r.m = rm[0];
      r.s = rs[0];
      r.s1 = rs1[0];
      for (int i = 1; i < DIS_WARPS; ++i) join<TWO>(r, rm[i], rs[i], rs1[i], ct, c1);
      if (!TWO) r.s1 = r.s;
    }
    const bool dead = w == 0.f || r.s == 0.f;  // nothing to learn: all -inf, or weight 0
    const float ls = logf(r.s);
    if (warp == 0) {
      float kd = 0.f;
      if (!dead) {
        for (int j = lane; j < A.K; j += 32) {
          const float q = eq[j];
          if (q != 0.f) kd += q * (elq[j] - ((ez[j] - r.m) / A.tau - ls));
        }
        kd = warp_sum(kd) * A.a * A.tau * A.tau;
        if (A.b != 0.f && hard) kd += A.b * (logf(r.s1) - (ez[A.K] - r.m));
        kd *= w;
      }
      if (lane == 0) A.loss[t] = kd;
    }
    if (dz) {
      const float qa = dead ? 0.f : w * A.a * A.tau;
      const float pa = dead ? 0.f : qa * msum / r.s;
      const float hb = dead || !hard ? 0.f : w * A.b;
      const float pb = dead || !hard ? 0.f : hb / r.s1;
      auto grad = [&](float v) {
        if (dead) return 0.f;
        return TWO ? pa * ex2((v - r.m) * ct) + pb * ex2((v - r.m) * c1) : (pa + pb) * ex2((v - r.m) * ct);
      };
      for (int p = tid; p < S.pieces; p += DIS_THREADS) {
        float v[N];
        const long at = S.head + (long)p * N;
        if (!dead) load<T, N>(z + at, v);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = grad(v[j]);
        if (same) store<T, N>(dz + at, v);
        else
          for (int j = 0; j < N; ++j) dz[at + j] = from_f32<T>(v[j]);
      }
      const int rest = A.V - S.head - S.pieces * N;
      if (tid < S.head + rest) {
        const int at = tid < S.head ? tid : A.V - rest + tid - S.head;
        dz[at] = from_f32<T>(grad(dead ? 0.f : to_f32(z[at])));
      }
      __syncthreads();
      if (!dead)
        for (int j = tid; j <= A.K; j += DIS_THREADS) {
          const int id = eid[j];
          if (id < 0) continue;
          float q = 0.f;
          for (int i = 0; i < A.K; ++i) q += eid[i] == id ? eq[i] : 0.f;
          dz[id] = from_f32<T>(grad(ez[j]) - qa * q - (id == label ? hb : 0.f));
        }
    }
    __syncthreads();  // the entries and the parts are free again
  }
}

}  // namespace
}  // namespace lx

extern "C" lx_status lx_distill_loss(int32_t dtype, const void* logits, int64_t ld, const int32_t* teacher_id,
                                     const float* teacher_logit, const float* teacher_lse, const int32_t* labels,
                                     const float* row_weight, int32_t T, int32_t V, int32_t K, float temperature,
                                     float kd_weight, float ce_weight, float* loss, void* dlogits, int64_t ldd,
                                     void* stream) {
  using namespace lx;
  if (dtype != LX_F32 && dtype != LX_BF16) return fail(LX_ERR_ARG, "unknown dtype");
  if (T < 0) return fail(LX_ERR_ARG, "T < 0");
  if (V < 1) return fail(LX_ERR_SHAPE, "V < 1");
  if (K < 1 || K > MAX_TEACHER) return fail(LX_ERR_ARG, "K must be in 1..LX_MAX_TEACHER");
  if (!(temperature > 0.f) || temperature > 3e38f) return fail(LX_ERR_ARG, "temperature must be positive and finite");
  if (ce_weight != 0.f && !labels) return fail(LX_ERR_ARG, "ce_weight needs labels");
  if (T == 0) return LX_OK;
  if (!logits || !teacher_id || !teacher_logit || !loss)
    return fail(LX_ERR_ARG, "logits, teacher_id, teacher_logit or loss is NULL");
  if (ld < V || (dlogits && ldd < V)) return fail(LX_ERR_SHAPE, "rows are closer than V elements");
  const size_t es = dtype == LX_BF16 ? 2 : 4;
  if (!aligned(logits, es) || !aligned(dlogits, es) || !aligned(teacher_id, 4) || !aligned(teacher_logit, 4) ||
      !aligned(teacher_lse, 4) || !aligned(labels, 4) || !aligned(row_weight, 4) || !aligned(loss, 4))
    return fail(LX_ERR_ARG, "a pointer is not aligned to its element");
  if (!(dlogits == logits && ldd == ld) && overlap(dlogits, span(T, V, ldd, es), logits, span(T, V, ld, es)))
    return fail(LX_ERR_ARG, "dlogits overlaps logits");
  DistillArgs A = {logits, ld, teacher_id, teacher_logit, teacher_lse, labels, row_weight, T, V, K,
                   temperature, kd_weight, ce_weight, loss, dlogits, ldd};
  const int grid = std::min(T, 152 * 4);
  cudaStream_t s = (cudaStream_t)stream;
  const bool two = ce_weight != 0.f && temperature != 1.f;
  if (dtype == LX_BF16) {
    if (two) k_distill<__nv_bfloat16, true><<<grid, DIS_THREADS, 0, s>>>(A);
    else k_distill<__nv_bfloat16, false><<<grid, DIS_THREADS, 0, s>>>(A);
  } else {
    if (two) k_distill<float, true><<<grid, DIS_THREADS, 0, s>>>(A);
    else k_distill<float, false><<<grid, DIS_THREADS, 0, s>>>(A);
  }
  LX_CUDA(cudaGetLastError());
  return LX_OK;
}
