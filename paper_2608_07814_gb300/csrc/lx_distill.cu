// Distillation from a teacher's stored top logits (lx_distill_loss).  For a token
// with student logits z [V], teacher entries (id_j, t_j), weight w:
//   q_j = softmax_j(t_j / tau) over the valid entries, or exp(t_j / tau - L),
//   kd  = sum_j q_j (log q_j - log p_{id_j}),  p = softmax(z / tau),  m = sum_j q_j
//   ce  = log sum_v exp z_v - z_label
//   loss = w (a tau^2 kd + b ce)
//   dz_v = w (a tau (m p_v - sum_{j: id_j = v} q_j) + b (softmax(z)_v - [v = label])).
//
// Bound by the logits: they are read from memory once and their gradient is written
// once.  A CTA (or a cluster of CTAs, where a row is long or rows are few) works on one row
// at a time.  Its threads hold their part of the row as 16-byte pieces in shared memory,
// each thread its own (cp.async, no barrier between copy and use).  The first pass over a
// row sums the exponentials against a running reference, one barrier joins the sums, the
// second pass writes the gradient.  The second pass of a row runs together with the first
// of the next one: a thread finishes a piece, asks for the one AHEAD + (pieces of a row)
// later in its place, and takes the next row's piece, which was asked for AHEAD pieces
// ago; reads and writes go on all the time (with the passes one after the other all CTAs
// drew on memory in the same halves of their rows: 489 us for 4096 rows of 131072 bf16).
// Rows that do not fit the shared memory of eight CTAs are read a second time from L2.  A
// warp of its own prepares the teacher's entries a row ahead.  The entries' places are
// written once more, behind the dense values, by the warp that wrote those; entries of
// one id add up.
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
constexpr int U = 2;               // pieces of a thread taken together
constexpr int AHEAD = 8;           // pieces asked for before they are used, a multiple of U
constexpr int REGS = 112;          // registers a thread: the launch bound holds the compiler to it
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
  int rounds; // pieces of a thread, rounded up to a multiple of U
  int slots;  // of them in shared memory at a time, a multiple of U
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Sums of 2^(z ct - n) and, with a second temperature, of 2^(z log2(e) - n1); p and p1
// are those of a pass that is under way, to be added
struct Run {
  float n = LOWEST, s = 0.f, n1 = LOWEST, s1 = 0.f;
  float2 p = {0.f, 0.f}, p1 = {0.f, 0.f};
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

// Adds the U pieces at q (those with `have` set) to sums p against reference n.  While the
// values lie less than 2^40 above the reference no maximum is needed; then it is raised
// to the pieces' maximum.
template <typename T>
__device__ __forceinline__ void add_pieces(float& n, float2& p, const uint4* q, float c) {
  constexpr int N2 = 8 / sizeof(T);
  auto sum = [&](float neg) {
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float2 v[N2];
      unpack<T>(q[u], v);
#pragma unroll
      for (int j = 0; j < N2; ++j) {
        const float2 x = fma2(v[j], both(c), both(neg));
        s = add2(s, make_float2(ex2(x.x), ex2(x.y)));
      }
    }
    return s;
  };
  float2 s = sum(-n);
  if (fmaxf(s.x, s.y) > 1099511627776.f) {  // (a NaN goes on as it is)
    float mx = piece_max<T>(q[0]);
    for (int u = 1; u < U; ++u) mx = fmaxf(mx, piece_max<T>(q[u]));
    const float N = ceilf(mx * c);
    p = mul2(p, both(ex2(n - N)));
    n = N;
    s = sum(-n);
  }
  p = add2(p, s);
}
__device__ __forceinline__ void add_value(float& n, float2& p, float v, float c) {
  const float t = v * c;
  if (t > n + 16.f) {
    const float N = ceilf(t);
    p = mul2(p, both(ex2(n - N)));
    n = N;
  }
  p.x += ex2(fmaf(v, c, -n));
}

extern __shared__ uint4 distill_smem[];

// TWO: a hard-label term at another temperature than the teacher's.  HELD: rows fit shared
// memory.  blockDim: the data threads and one warp more, which prepares the entries;
// gridDim: (CTAs of a row, rows)
template <typename T, bool TWO, bool CL, bool HELD>
__global__ void __launch_bounds__(576, 1)
k_distill(const __grid_constant__ DistillArgs A) {
  constexpr int N = Span<T>::N, N2 = N / 2;
  __shared__ float4 red[2][CL ? MAX_CLUSTER : 1][MAX_WARPS];
  __shared__ float msum[2];
  const int D = blockDim.x - 32, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = D >> 5;
  const bool teacher = warp == nw, grad = A.dlogits != nullptr;
  const int E1 = A.K + 1, rank = CL ? blockIdx.x : 0, cols = CL ? gridDim.x : 1;
  // entries of the row and of the next: id, z, q, log q; entry K is the label
  int* eid = (int*)distill_smem;
  float* ez = (float*)distill_smem + 2 * E1;
  float* eq = ez + 2 * E1;
  float* elq = eq + 2 * E1;
  const uint4* slot = distill_smem + (8 * E1 + 3) / 4 + tid;  // slot k at slot[k * D]
  const uint32_t slot_at = (uint32_t)__cvta_generic_to_shared(slot);
  const int v0 = rank * A.slice, vn = min(A.slice, A.V - v0);
  const float ct = A.ct;
  const long first = blockIdx.y, step = gridDim.y;
  auto weight = [&](long t) { return t >= A.T ? 0.f : A.weight ? A.weight[t] : 1.f; };
  auto span = [&](long t) { return Span<T>((const T*)A.logits + (t < A.T ? t : first) * A.ld + v0, vn); };
  // the copies, U pieces a group, in the order of use: rows of weight 0 and pieces that a
  // thread does not have leave their slots as they are
  auto mine = [&](const Span<T>& S) { return (S.pieces - tid + D - 1) / D; };
  long ask_t = first;
  float ask_wn = weight(first);
  const T* ask_at = nullptr;
  int ask_left = 0, ask_rounds = 0;  // pieces of the thread, rounds of the row not asked for yet
  auto ask = [&](uint32_t to) {
    if (ask_rounds == 0) {
      const Span<T> S = span(ask_t);
      ask_at = S.piece(tid);
      ask_left = ask_wn != 0.f ? mine(S) : 0;
      ask_rounds = A.rounds;
      ask_t += step;
      ask_wn = weight(ask_t);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u < ask_left)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slot_at + to + u * D * 16), "l"(ask_at + (long)u * D * N)
                     : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
    ask_at += (long)U * D * N;
    ask_left -= U;
    ask_rounds -= U;
  };
  const uint32_t batch = U * D * 16, ring = A.slots * D * 16;  // bytes
  auto advance = [&](uint32_t& k) { k = k + batch == ring ? 0 : k + batch; };
  // U pieces from slot offset k, -inf (which adds nothing) where the thread has fewer
  auto fetch = [&](uint32_t k, int have, uint4* q) {
    const uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
    for (int u = 0; u < U; ++u)
      q[u] = u < have ? *(const uint4*)((const char*)slot + k + u * D * 16) : make_uint4(none, none, none, none);
  };
  // the CTAs of the row meet
  auto meet = [&] {
    if constexpr (CL) cooperative_groups::this_cluster().sync();
    else __syncthreads();
  };
  // joins the threads' sums over the row; the same in every thread (the teacher's too)
  int turn = 0;
  auto joined = [&](Run r) {
    r.s += r.p.x + r.p.y;
    if (TWO) r.s1 += r.p1.x + r.p1.y;
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

  // the first pass: U pieces of the thread into the sums
  auto take = [&](Run& r, const uint4* q) {
    add_pieces<T>(r.n, r.p, q, ct);
    if (TWO) add_pieces<T>(r.n1, r.p1, q, LOG2E);
  };
  auto take_edge = [&](Run& r, float v) {
    add_value(r.n, r.p, v, ct);
    if (TWO) add_value(r.n1, r.p1, v, LOG2E);
  };
  auto landed = [] { asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD / U) : "memory"); };
  uint32_t k0 = 0, k1 = 0;  // slot offsets of the copies and of the first pass
  // the first pass of a whole row by itself: the first row, and every row without gradient
  auto pass1 = [&](const Span<T>& S, float w, Run& r) {
    const int n = w != 0.f ? mine(S) : 0;
    uint4 q[U];
    if constexpr (HELD) {
      for (int p = 0; p < A.rounds; p += U) {
        ask(k0);
        advance(k0);
        landed();
        if (p < n) {
          fetch(k1, n - p, q);
          take(r, q);
        }
        advance(k1);
      }
    } else {
      const uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
      for (int p = 0; p < n; p += U) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          q[u] = p + u < n ? *(const uint4*)S.piece((p + u) * D + tid) : make_uint4(none, none, none, none);
        take(r, q);
      }
    }
    if (w != 0.f && tid < S.edges) take_edge(r, to_f32(S.row[S.edge(tid)]));
  };

  float w = weight(first), wn = weight(first + step);
  Run r;
  if (teacher) {
    prepare(first, 0);
  } else {
    if constexpr (HELD)
      for (int p = 0; p < AHEAD; p += U) {
        ask(k0);
        advance(k0);
      }
    pass1(span(first), w, r);
  }
  if constexpr (CL) cooperative_groups::this_cluster().sync();  // all have started
  int half = 0;
  uint32_t k2 = 0;  // slot offset of the second pass
  for (long t = first; t < A.T; t += step, half ^= 1) {
    const Span<T> S = span(t), Sn = span(t + step);
    const float wn2 = weight(t + 2 * step);
    bool slow = false, dead = w == 0.f;  // dead: nothing to learn
    float top = 0.f;                     // slow: the row's maximum
    if (!dead) {
      r = joined(r);
      if (r.s == 0.f) {  // every logit is -inf or out of the references' reach
        slow = true;
        top = -INFINITY;
        if (!teacher) {
          for (int i = tid; i < S.pieces; i += D) top = fmaxf(top, piece_max<T>(*(const uint4*)S.piece(i)));
          if (tid < S.edges) top = fmaxf(top, to_f32(S.row[S.edge(tid)]));
        }
        auto max_of = [&](float x) {
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
          return x;
        };
        top = max_of(top);
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
    }
    // z relative to the references, in powers of two
    auto rel = [&](float z) { return slow ? (z - top) * ct : fmaf(z, ct, -r.n); };
    auto rel1 = [&](float z) { return slow ? (z - top) * LOG2E : fmaf(z, LOG2E, -r.n1); };
    const int* id = eid + half * E1;
    const float *zj = ez + half * E1, *q = eq + half * E1, *lq = elq + half * E1;
    Run rn;  // the next row's sums
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
    } else if (!grad) {
      if (t + step < A.T) pass1(Sn, wn, rn);
    } else {
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
      const float2 pa2 = both(TWO ? pa : pa + pb), pb2 = both(pb), nn = both(-r.n), nn1 = both(-r.n1);
      auto gradient = [&](uint4 w4) {
        float2 v[N2];
        unpack<T>(w4, v);
#pragma unroll
        for (int j = 0; j < N2; ++j) {
          const float2 x = fma2(v[j], both(ct), nn);
          float2 o = mul2(make_float2(ex2(x.x), ex2(x.y)), pa2);
          if (TWO) {
            const float2 x1 = fma2(v[j], both(LOG2E), nn1);
            o = fma2(make_float2(ex2(x1.x), ex2(x1.y)), pb2, o);
          }
          v[j] = o;
        }
        if constexpr (sizeof(T) == 4)
          return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x),
                            __float_as_uint(v[1].y));
        else
          return make_uint4(to_bf2(v[0]), to_bf2(v[1]), to_bf2(v[2]), to_bf2(v[3]));
      };
      // a piece of a row that is dead or slow, or whose gradient lies at other addresses
      auto odd_piece = [&](const uint4* from, T* out) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (!dead) {
          x = *from;
          if (slow) {
            float2 v[N2];
            unpack<T>(x, v);
            alignas(16) T o[N];
#pragma unroll
            for (int j = 0; j < N2; ++j) {
              o[2 * j] = from_f32<T>(value(v[j].x));
              o[2 * j + 1] = from_f32<T>(value(v[j].y));
            }
            x = *(const uint4*)o;
          } else {
            x = gradient(x);
          }
        }
        if (same) {
          *(uint4*)out = x;
        } else {
          const T* o = (const T*)&x;
#pragma unroll
          for (int j = 0; j < N; ++j) out[j] = o[j];
        }
      };
      T* out = dz + S.head + (long)tid * N;
      const int n = mine(S), nn_row = wn != 0.f ? mine(Sn) : 0;
      const bool plain = same && !slow && !dead;
      if constexpr (HELD) {
        const float en = wn != 0.f && tid < Sn.edges ? to_f32(Sn.row[Sn.edge(tid)]) : 0.f;
        // the thread's batches that are whole in both rows, and the rest
        const int full = plain ? min(n, nn_row) / U * U : 0;
        int p = 0;
        uint4 x[U];
        for (; p < full; p += U) {
#pragma unroll
          for (int u = 0; u < U; ++u) x[u] = *(const uint4*)((const char*)slot + k2 + u * D * 16);
#pragma unroll
          for (int u = 0; u < U; ++u) *(uint4*)(out + (long)u * D * N) = gradient(x[u]);
          ask(k2);  // the values have been used: the place is free
          advance(k2);
          landed();
#pragma unroll
          for (int u = 0; u < U; ++u) x[u] = *(const uint4*)((const char*)slot + k1 + u * D * 16);
          take(rn, x);
          advance(k1);
          out += (long)U * D * N;
        }
        for (; p < A.rounds; p += U) {
          for (int u = 0; u < U && p + u < n; ++u)
            odd_piece((const uint4*)((const char*)slot + k2 + u * D * 16), out + (long)u * D * N);
          ask(k2);
          advance(k2);
          landed();
          if (p < nn_row) {
            fetch(k1, nn_row - p, x);
            take(rn, x);
          }
          advance(k1);
          out += (long)U * D * N;
        }
        if (wn != 0.f && tid < Sn.edges) take_edge(rn, en);
      } else {
        for (int p = 0; p < n; ++p, out += (long)D * N) {
          const uint4* from = (const uint4*)S.piece(p * D + tid);
          if (plain) *(uint4*)out = gradient(*from);
          else odd_piece(from, out);
        }
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
      if constexpr (!HELD)
        if (t + step < A.T) pass1(Sn, wn, rn);
    }
    r = rn;
    w = wn;
    wn = wn2;
  }
  // shared memory outlives the copies and the neighbours' writes
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  if constexpr (CL) cooperative_groups::this_cluster().sync();
}

template <typename T, bool TWO, bool CL, bool HELD>
lx_status launch_distill(const DistillArgs& A, int threads, int cols, int groups, size_t smem, cudaStream_t s) {
  static bool cap[64] = {};
  int dev = 0;
  LX_CUDA(cudaGetDevice(&dev));
  LX_CUDA(smem_cap_once((const void*)k_distill<T, TWO, CL, HELD>, SMEM, dev, cap));
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
  LX_CUDA(cudaLaunchKernelEx(&cfg, k_distill<T, TWO, CL, HELD>, A));
  return LX_OK;
}

template <typename T, bool CL, bool HELD>
lx_status launch_two(const DistillArgs& A, bool two, int threads, int cols, int groups, size_t smem, cudaStream_t s) {
  return two ? launch_distill<T, true, CL, HELD>(A, threads, cols, groups, smem, s)
             : launch_distill<T, false, CL, HELD>(A, threads, cols, groups, smem, s);
}
template <typename T>
lx_status launch_type(const DistillArgs& A, bool two, int threads, int cols, int groups, size_t smem, cudaStream_t s) {
  if (A.slots == 0) return launch_two<T, false, false>(A, two, threads, cols, groups, smem, s);
  if (cols > 1) return launch_two<T, true, true>(A, two, threads, cols, groups, smem, s);
  return launch_two<T, false, true>(A, two, threads, cols, groups, smem, s);
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
  // Data threads that hold `bytes` of a row, and the CTAs of a row: as many as it takes to
  // hold it, and more where rows are few, in slices of 4096 columns at least
  const size_t entries = ((8 * (size_t)(K + 1) + 3) / 4) * 16;
  const int most = ((int)((SMEM - entries) / (16 * 512)) - AHEAD) / U * U;  // pieces of each of 512 threads
  const long row = (long)V * es;
  int cols = 1;
  while (cols < MAX_CLUSTER && row > 16L * 512 * most * cols) cols *= 2;
  const bool held = row <= 16L * 512 * most * cols;
  if (!held) cols = 1;
  else
    while (cols < MAX_CLUSTER && (long)T * cols * 2 <= SMS && V / (cols * 2) >= 4096) cols *= 2;
  A.slice = cols == 1 ? V : ((V + cols - 1) / cols + 63) / 64 * 64;
  const long bytes = (long)A.slice * es;
  const int threads = bytes > 16L * 256 * most ? 512 : bytes > 16L * 128 * most ? 256 : 128;
  A.rounds = (int)((bytes / 16 + threads - 1) / threads + U - 1) / U * U;
  if (A.rounds == 0) A.rounds = U;
  A.slots = !held ? 0 : dlogits ? A.rounds + AHEAD : AHEAD + U;
  const size_t smem = entries + (size_t)16 * threads * A.slots;
  const int ctas = std::max(1, std::min((int)(65536 / (REGS * (threads + 32))), (int)(227 * 1024 / (smem + 5120))));
  const int groups = std::min(T, std::max(1, SMS * ctas / cols));
  const bool two = ce_weight != 0.f && temperature != 1.f;
  cudaStream_t s = (cudaStream_t)stream;
  return dtype == LX_BF16 ? launch_type<__nv_bfloat16>(A, two, threads, cols, groups, smem, s)
                          : launch_type<float>(A, two, threads, cols, groups, smem, s);
}
