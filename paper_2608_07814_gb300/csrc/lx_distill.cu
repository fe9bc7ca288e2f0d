// Distillation from a teacher's stored top logits (lx_distill_loss).  For a token
// with student logits z [V], teacher entries (id_j, t_j), weight w:
//   q_j = softmax_j(t_j / tau) over the valid entries, or exp(t_j / tau - L),
//   kd  = sum_j q_j (log q_j - log p_{id_j}),  p = softmax(z / tau),  m = sum_j q_j
//   ce  = log sum_v exp z_v - z_label
//   loss = w (a tau^2 kd + b ce)
//   dz_v = w (a tau (m p_v - sum_{j: id_j = v} q_j) + b (softmax(z)_v - [v = label])).
//
// Bound by the logits: they are read from memory once and their gradient is written
// once.  A CTA (or a cluster of CTAs, where rows are few) works on one row at a time.  Its
// threads hold the row as 16-byte pieces in shared memory, each thread its own (cp.async,
// no barrier), as far as they fit; the rest of a long row is read a second time from L2,
// which holds a row for each SM.  The first pass over the pieces sums the exponentials
// against a running reference, one barrier joins the sums, the second pass writes the
// gradient and asks for the next row's piece in each place that it leaves.  A warp of its
// own prepares the teacher's entries a row ahead.  The entries' places are written once
// more, behind the dense values, by the warp that wrote those; entries of one id add up.
//
// The reference of a sum is a whole number n of powers of two: exp(z / tau) is taken as
// 2^n 2^(z log2(e) / tau - n), one fused multiply-add from z, exact in n, and partial sums
// are joined by powers of two without rounding.  A row whose every logit lies below -2^30
// powers of two sums to zero against the lowest reference and is done again with its
// maximum subtracted first.
#include <algorithm>

#include "lx_rows.cuh"

namespace lx {
namespace {

using namespace rows;

constexpr int SMS = 152;
constexpr int MAX_WARPS = 16;      // data warps of a CTA
constexpr int MAX_CLUSTER = 8;
constexpr int SMEM = 222 * 1024;   // dynamic shared memory of a CTA at most
constexpr float LOWEST = -1073741824.f;  // -2^30
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct DistillArgs {
  const void* logits;
  long ld;
  const int* ids;
  const float* top;
  const float* top_lse;
  const int* labels;
  const float* weight;
  int T, V, K;
  float tau, ct, a, b;  // ct: log2(e) / tau
  float* loss;
  void* dlogits;
  long ldd;
  int slice;  // columns of a CTA
  int slots;  // pieces of a thread in shared memory
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Sums of 2^(z ct - n) and, with a second temperature, of 2^(z log2(e) - n1)
struct Run {
  float n = LOWEST, s = 0.f, n1 = LOWEST, s1 = 0.f;
};
__device__ __forceinline__ void join(float& n, float& s, float on, float os) {
  const float N = fmaxf(n, on);
  s = s * ex2(n - N) + os * ex2(on - N);
  n = N;
}
template <bool TWO>
__device__ __forceinline__ void join(Run& r, float4 o) {
  join(r.n, r.s, o.x, o.y);
  if (TWO) join(r.n1, r.s1, o.z, o.w);
}

// A row part: elements before its first 16-byte boundary, 16-byte pieces, the rest
template <typename T>
struct Span {
  static constexpr int N = 16 / sizeof(T);
  const T* row;
  int head, pieces, edges;  // edges: elements outside the pieces
  __device__ Span(const T* p, int n) : row(p) {
    head = min(n, (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T));
    pieces = (n - head) / N;
    edges = n - pieces * N;
  }
  __device__ const T* piece(int i) const { return row + head + (long)i * N; }
  __device__ int edge(int i) const { return i < head ? i : i + pieces * N; }  // place of edge i
};

template <typename T>
__device__ __forceinline__ void unpack(uint4 w, float2* v) {
  if constexpr (sizeof(T) == 4) {
    v[0] = make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
    v[1] = make_float2(__uint_as_float(w.z), __uint_as_float(w.w));
  } else {
    v[0] = bf2(w.x);
    v[1] = bf2(w.y);
    v[2] = bf2(w.z);
    v[3] = bf2(w.w);
  }
}
template <typename T>
__device__ __forceinline__ float piece_max(uint4 w) {  // a NaN is left out: it shows in the sums
  if constexpr (sizeof(T) == 4) {
    return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
  } else {
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&w);
    const __nv_bfloat162 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
    return fmaxf(__low2float(m), __high2float(m));
  }
}

// Raises a reference that the values of a batch with maximum mx are far above
__device__ __forceinline__ void raise(float& n, float& s, float t) {
  if (t > n + 16.f) {
    const float N = ceilf(t);
    s *= ex2(n - N);
    n = N;
  }
}

extern __shared__ uint4 distill_smem[];

// TWO: a hard-label term at another temperature than the teacher's.  blockDim: the data
// threads and one warp more, which prepares the entries; gridDim: (CTAs of a row, rows)
template <typename T, bool TWO, bool CL>
__global__ void __launch_bounds__(896, 1)
k_distill(const __grid_constant__ DistillArgs A) {
  constexpr int N = Span<T>::N, N2 = N / 2;
  __shared__ float4 red[2][CL ? MAX_CLUSTER : 1][MAX_WARPS];
  __shared__ float msum[2];
  const int D = blockDim.x - 32, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = D >> 5;
  const bool teacher = warp == nw;
  const int E1 = A.K + 1, rank = CL ? blockIdx.x : 0, cols = CL ? gridDim.x : 1;
  // entries of the row and of the next: id, z, q, log q; entry K is the label
  int* eid = (int*)distill_smem;
  float* ez = (float*)distill_smem + 2 * E1;
  float* eq = ez + 2 * E1;
  float* elq = eq + 2 * E1;
  uint4* slot = distill_smem + (8 * E1 + 3) / 4 + tid;  // piece p at slot[p * D]
  const int v0 = rank * A.slice, vn = min(A.slice, A.V - v0);
  const float ct = A.ct;
  auto weight = [&](long t) { return t >= A.T ? 0.f : A.weight ? A.weight[t] : 1.f; };
  auto span = [&](long t) { return Span<T>((const T*)A.logits + t * A.ld + v0, vn); };
  auto ask = [&](const Span<T>& S, int p) {
    const int i = p * D + tid;
    if (i < S.pieces)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(slot + p * D)),
                   "l"(S.piece(i))
                   : "memory");
  };
  auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
  // the CTAs of the row meet
  auto meet = [&] {
    if constexpr (CL) cooperative_groups::this_cluster().sync();
    else __syncthreads();
  };
  // joins the threads' sums over the row; the same in every thread (the teacher's too)
  int turn = 0;
  auto joined = [&](Run r) {
    if (!teacher) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        join<TWO>(r, make_float4(__shfl_xor_sync(0xffffffffu, r.n, o), __shfl_xor_sync(0xffffffffu, r.s, o),
                                 TWO ? __shfl_xor_sync(0xffffffffu, r.n1, o) : 0.f,
                                 TWO ? __shfl_xor_sync(0xffffffffu, r.s1, o) : 0.f));
      const float4 mine = make_float4(r.n, r.s, r.n1, r.s1);
      if constexpr (CL) {
        if (lane < cols) *cooperative_groups::this_cluster().map_shared_rank(&red[turn][rank][warp], lane) = mine;
      } else {
        if (lane == 0) red[turn][0][warp] = mine;
      }
    }
    meet();
    r = Run();
    for (int i = lane; i < cols * MAX_WARPS; i += 32)
      if ((i & (MAX_WARPS - 1)) < nw) join<TWO>(r, red[turn][i / MAX_WARPS][i & (MAX_WARPS - 1)]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      join<TWO>(r, make_float4(__shfl_xor_sync(0xffffffffu, r.n, o), __shfl_xor_sync(0xffffffffu, r.s, o),
                               TWO ? __shfl_xor_sync(0xffffffffu, r.n1, o) : 0.f,
                               TWO ? __shfl_xor_sync(0xffffffffu, r.s1, o) : 0.f));
    turn ^= 1;
    return r;
  };

  // the teacher's entries of row t into half `half`
  auto prepare = [&](long t, int half) {
    if (weight(t) == 0.f) return;
    int* id = eid + half * E1;
    float *z = ez + half * E1, *q = eq + half * E1, *lq = elq + half * E1;
    const T* row = (const T*)A.logits + t * A.ld;
    float tm = -INFINITY;
    for (int j = lane; j < A.K; j += 32) {
      const int e = A.ids[t * A.K + j];
      const bool ok = e >= 0 && e < A.V;
      const float v = ok ? A.top[t * A.K + j] : -INFINITY;
      id[j] = ok ? e : -1;
      z[j] = ok ? to_f32(row[e]) : 0.f;
      q[j] = v;
      tm = fmaxf(tm, v);
    }
    if (lane == 0) {
      const int e = A.labels ? A.labels[t] : -1;
      const bool ok = e >= 0 && e < A.V;
      id[A.K] = ok ? e : -1;
      z[A.K] = ok ? to_f32(row[e]) : 0.f;
      q[A.K] = 0.f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) tm = fmaxf(tm, __shfl_xor_sync(0xffffffffu, tm, o));
    float lz;  // log of the distribution's sum, relative to tm / tau
    if (A.top_lse) {
      lz = A.top_lse[t] - tm / A.tau;
    } else {
      float s = 0.f;
      for (int j = lane; j < A.K; j += 32)
        if (id[j] >= 0) s += tm == -INFINITY ? 0.f : expf((q[j] - tm) / A.tau);
      lz = logf(warp_sum(s));
    }
    float m = 0.f;
    for (int j = lane; j < A.K; j += 32) {
      const float l = id[j] >= 0 && q[j] != -INFINITY ? (q[j] - tm) / A.tau - lz : -INFINITY;
      const float p = expf(l);
      lq[j] = l;
      q[j] = p;
      m += p;
    }
    m = warp_sum(m);
    if (lane == 0) msum[half] = m;
  };

  const long first = blockIdx.y, step = gridDim.y;
  float w = weight(first);
  if (teacher) {
    prepare(first, 0);
  } else if (w != 0.f) {
    const Span<T> S = span(first);
    for (int p = 0; p < A.slots; ++p) ask(S, p);
  }
  commit();
  if constexpr (CL) cooperative_groups::this_cluster().sync();  // all have started
  int half = 0;
  for (long t = first; t < A.T; t += step, half ^= 1) {
    const float wn = weight(t + step);
    const Span<T> S = span(t), Sn = span(t + step < A.T ? t + step : t);
    const bool grad = A.dlogits != nullptr, ahead = wn != 0.f;
    const int rounds = (S.pieces + D - 1) / D, held = min(rounds, A.slots);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    Run r;
    bool slow = false, dead = w == 0.f;  // dead: nothing to learn
    float top = 0.f;                     // slow: the row's maximum
    if (!dead) {
      if (!teacher) {
        auto take = [&](const uint4* q, int n) {  // n pieces, all inside the row
          float mx = piece_max<T>(q[0]);
          for (int u = 1; u < n; ++u) mx = fmaxf(mx, piece_max<T>(q[u]));
          raise(r.n, r.s, mx * ct);
          if (TWO) raise(r.n1, r.s1, mx * LOG2E);
          float2 s = make_float2(0.f, 0.f), s1 = s;
          for (int u = 0; u < n; ++u) {
            float2 v[N2];
            unpack<T>(q[u], v);
#pragma unroll
            for (int j = 0; j < N2; ++j) {
              const float2 x = fma2(v[j], both(ct), both(-r.n));
              s = add2(s, make_float2(ex2(x.x), ex2(x.y)));
              if (TWO) {
                const float2 x1 = fma2(v[j], both(LOG2E), both(-r.n1));
                s1 = add2(s1, make_float2(ex2(x1.x), ex2(x1.y)));
              }
            }
          }
          r.s += s.x + s.y;
          if (TWO) r.s1 += s1.x + s1.y;
        };
        const int mine = (S.pieces - tid + D - 1) / D;  // the thread's pieces
        constexpr int U = 4;
        int p = 0;
        for (; p + U <= mine; p += U) {
          uint4 q[U];
#pragma unroll
          for (int u = 0; u < U; ++u)
            q[u] = p + u < held ? slot[(p + u) * D] : *(const uint4*)S.piece((p + u) * D + tid);
          take(q, U);
          if (!grad && ahead)
            for (int u = 0; u < U; ++u)
              if (p + u < A.slots) ask(Sn, p + u);
        }
        for (; p < mine; ++p) {
          const uint4 q = p < held ? slot[p * D] : *(const uint4*)S.piece(p * D + tid);
          take(&q, 1);
          if (!grad && ahead && p < A.slots) ask(Sn, p);
        }
        if (!grad && ahead)
          for (; p < A.slots; ++p) ask(Sn, p);  // a row with a piece more
        if (tid < S.edges) {
          const float v = to_f32(S.row[S.edge(tid)]);
          raise(r.n, r.s, v * ct);
          r.s += ex2(fmaf(v, ct, -r.n));
          if (TWO) {
            raise(r.n1, r.s1, v * LOG2E);
            r.s1 += ex2(fmaf(v, LOG2E, -r.n1));
          }
        }
      }
      r = joined(r);
      if (r.s == 0.f) {  // every logit is -inf or out of the references' reach
        slow = true;
        Run m;  // n: the maximum
        m.n = -INFINITY;
        if (!teacher) {
          for (int i = tid; i < S.pieces; i += D) m.n = fmaxf(m.n, piece_max<T>(*(const uint4*)S.piece(i)));
          if (tid < S.edges) m.n = fmaxf(m.n, to_f32(S.row[S.edge(tid)]));
        }
        // (the sums of this round are zero: the reference that comes out is the maximum,
        // or LOWEST where that is below it)
        auto max_of = [&](float x) {
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
          return x;
        };
        top = max_of(m.n);
        if (!teacher) {
          if constexpr (CL) {
            if (lane < cols) cooperative_groups::this_cluster().map_shared_rank(&red[turn][rank][warp], lane)->x = top;
          } else {
            if (lane == 0) red[turn][0][warp].x = top;
          }
        }
        meet();
        top = -INFINITY;
        for (int i = lane; i < cols * MAX_WARPS; i += 32)
          if ((i & (MAX_WARPS - 1)) < nw) top = fmaxf(top, red[turn][i / MAX_WARPS][i & (MAX_WARPS - 1)].x);
        top = max_of(top);
        turn ^= 1;
        dead = top == -INFINITY;
        if (!dead) {
          r = Run();
          r.n = r.n1 = 0.f;
          if (!teacher) {
            auto add = [&](float v) {
              r.s += ex2((v - top) * ct);
              if (TWO) r.s1 += ex2((v - top) * LOG2E);
            };
            for (int i = tid; i < S.pieces * N; i += D) add(to_f32(S.row[S.head + i]));
            if (tid < S.edges) add(to_f32(S.row[S.edge(tid)]));
          }
          r = joined(r);
        }
      }
      if (!TWO) r.n1 = r.n, r.s1 = r.s;
    } else {
      __syncthreads();  // the entries' other half is free for the teacher's warp
      if (!teacher && !grad && ahead)
        for (int p = 0; p < A.slots; ++p) ask(Sn, p);
    }
    // z relative to the references, in powers of two
    auto rel = [&](float z) { return slow ? (z - top) * ct : fmaf(z, ct, -r.n); };
    auto rel1 = [&](float z) { return slow ? (z - top) * LOG2E : fmaf(z, LOG2E, -r.n1); };
    const int* id = eid + half * E1;
    const float *zj = ez + half * E1, *q = eq + half * E1, *lq = elq + half * E1;
    if (teacher) {
      float loss = 0.f;
      if (!dead) {
        const float ls = logf(r.s);
        for (int j = lane; j < A.K; j += 32)
          if (q[j] != 0.f) loss += q[j] * (lq[j] - (rel(zj[j]) * LN2 - ls));
        loss = warp_sum(loss) * A.a * A.tau * A.tau;
        if (A.b != 0.f && id[A.K] >= 0) loss += A.b * (logf(r.s1) - (TWO ? rel1(zj[A.K]) : rel(zj[A.K])) * LN2);
        loss *= w;
      }
      if (lane == 0 && rank == 0) A.loss[t] = loss;
      if (t + step < A.T) prepare(t + step, half ^ 1);
    } else if (grad) {
      T* dz = (T*)A.dlogits + t * A.ldd + v0;
      const bool same = (((uintptr_t)dz ^ (uintptr_t)S.row) & 15) == 0;
      const int label = dead ? -1 : id[A.K];
      const float qa = dead ? 0.f : w * A.a * A.tau;
      const float hb = dead || label < 0 ? 0.f : w * A.b;
      const float pa = dead ? 0.f : qa * msum[half] / r.s, pb = dead ? 0.f : hb / r.s1;
      auto value = [&](float z) {
        if (dead) return 0.f;
        return TWO ? pa * ex2(rel(z)) + pb * ex2(rel1(z)) : (pa + pb) * ex2(rel(z));
      };
      const int mine = (S.pieces - tid + D - 1) / D;
      const float2 pa2 = both(TWO ? pa : pa + pb), pb2 = both(pb);
      for (int p = 0; p < max(mine, A.slots); ++p) {
        if (p < mine) {
          float2 v[N2];
          const long at = S.head + (long)(p * D + tid) * N;
          if (dead) {
#pragma unroll
            for (int j = 0; j < N2; ++j) v[j] = make_float2(0.f, 0.f);
          } else {
            unpack<T>(p < held ? slot[p * D] : *(const uint4*)S.piece(p * D + tid), v);
            if (slow) {
#pragma unroll
              for (int j = 0; j < N2; ++j) v[j] = make_float2(value(v[j].x), value(v[j].y));
            } else {
#pragma unroll
              for (int j = 0; j < N2; ++j) {
                const float2 x = fma2(v[j], both(ct), both(-r.n));
                float2 o = mul2(make_float2(ex2(x.x), ex2(x.y)), pa2);
                if (TWO) {
                  const float2 x1 = fma2(v[j], both(LOG2E), both(-r.n1));
                  o = fma2(make_float2(ex2(x1.x), ex2(x1.y)), pb2, o);
                }
                v[j] = o;
              }
            }
          }
          if (same) {
            uint4 o;
            if constexpr (sizeof(T) == 4)
              o = make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x),
                             __float_as_uint(v[1].y));
            else
              o = make_uint4(to_bf2(v[0]), to_bf2(v[1]), to_bf2(v[2]), to_bf2(v[3]));
            *(uint4*)(dz + at) = o;
          } else {
#pragma unroll
            for (int j = 0; j < N2; ++j) {
              dz[at + 2 * j] = from_f32<T>(v[j].x);
              dz[at + 2 * j + 1] = from_f32<T>(v[j].y);
            }
          }
        }
        if (ahead && p < A.slots) ask(Sn, p);  // its values have been used: the place is free
      }
      if (tid < S.edges) dz[S.edge(tid)] = from_f32<T>(value(dead ? 0.f : to_f32(S.row[S.edge(tid)])));
      __syncwarp();
      if (!dead)  // the entries that lie among this warp's values
        for (int j = lane; j <= A.K; j += 32) {
          const int e = id[j] - v0;
          if (id[j] < 0 || e < 0 || e >= vn) continue;
          const int i = e - S.head;
          const bool piece = i >= 0 && i < S.pieces * N;
          if ((piece ? i / N % D : i < 0 ? e : e - S.pieces * N) / 32 != warp) continue;
          float x = 0.f;
          for (int k = 0; k < A.K; ++k) x += id[k] == id[j] ? q[k] : 0.f;
          dz[e] = from_f32<T>(value(zj[j]) - qa * x - (id[j] == label ? hb : 0.f));
        }
    }
    commit();
    w = wn;
  }
  // shared memory outlives the copies and the neighbours' writes
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  if constexpr (CL) cooperative_groups::this_cluster().sync();
}

template <typename T, bool TWO, bool CL>
lx_status launch_distill(const DistillArgs& A, int threads, int cols, int groups, size_t smem, cudaStream_t s) {
  static bool cap[64] = {};
  int dev = 0;
  LX_CUDA(cudaGetDevice(&dev));
  LX_CUDA(smem_cap_once((const void*)k_distill<T, TWO, CL>, SMEM, dev, cap));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cols, groups);
  cfg.blockDim = dim3(threads + 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cols;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CL ? 1 : 0;
  LX_CUDA(cudaLaunchKernelEx(&cfg, k_distill<T, TWO, CL>, A));
  return LX_OK;
}

template <typename T>
lx_status launch_type(const DistillArgs& A, bool two, int threads, int cols, int groups, size_t smem, cudaStream_t s) {
  if (cols > 1)
    return two ? launch_distill<T, true, true>(A, threads, cols, groups, smem, s)
               : launch_distill<T, false, true>(A, threads, cols, groups, smem, s);
  return two ? launch_distill<T, true, false>(A, threads, cols, groups, smem, s)
             : launch_distill<T, false, false>(A, threads, cols, groups, smem, s);
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
  if (K < 1 || K > LX_MAX_TEACHER) return fail(LX_ERR_ARG, "K must be in 1..LX_MAX_TEACHER");
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
  DistillArgs A = {};
  A.logits = logits;
  A.ld = ld;
  A.ids = teacher_id;
  A.top = teacher_logit;
  A.top_lse = teacher_lse;
  A.labels = labels;
  A.weight = row_weight;
  A.T = T;
  A.V = V;
  A.K = K;
  A.tau = temperature;
  A.ct = (float)(1.4426950408889634 / (double)temperature);
  A.a = kd_weight;
  A.b = ce_weight;
  A.loss = loss;
  A.dlogits = dlogits;
  A.ldd = ldd;
  // Few rows are split over a cluster, in slices of 4096 columns at least
  int cols = 1;
  while (cols < MAX_CLUSTER && (long)T * cols * 2 <= SMS && V / (cols * 2) >= 4096) cols *= 2;
  A.slice = cols == 1 ? V : ((V + cols - 1) / cols + 63) / 64 * 64;
  const long bytes = (long)A.slice * es;
  const int threads = bytes > 100 * 1024 ? 512 : bytes > 24 * 1024 ? 256 : 128;
  const size_t entries = ((8 * (size_t)(K + 1) + 3) / 4) * 16;
  const long want = (bytes / 16 + threads - 1) / threads;
  A.slots = (int)std::min<long>(want, (long)(SMEM - entries) / (16 * threads));
  const size_t smem = entries + (size_t)16 * threads * A.slots;
  const int ctas = std::max(1, std::min((int)(65536 / (72 * (threads + 32))), (int)(227 * 1024 / (smem + 4096))));
  const int groups = std::min(T, std::max(1, SMS * ctas / cols));
  const bool two = ce_weight != 0.f && temperature != 1.f;
  cudaStream_t s = (cudaStream_t)stream;
  return dtype == LX_BF16 ? launch_type<__nv_bfloat16>(A, two, threads, cols, groups, smem, s)
                          : launch_type<float>(A, two, threads, cols, groups, smem, s);
}
