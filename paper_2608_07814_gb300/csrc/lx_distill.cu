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
// row sums the exponentials against a running reference, an exchange joins the sums, the
// second pass writes the gradient.  The second pass of a row runs together with the first
// of the next one: a thread finishes a batch of pieces, asks for the ones AHEAD + (pieces
// of a row) later in their place, and takes the next row's batch, which was asked for AHEAD
// pieces ago; reads and writes go on all the time (with the passes one after the other all
// CTAs drew on memory in the same halves of their rows).  Rows that do not fit the shared
// memory of eight CTAs are read a second time from L2.
//
// Two warps of their own prepare the teacher's entries, up to four rows ahead, and write the
// losses: their chains of loads take longer than a row.  The entries' places are written
// once more, behind the dense values, by the warp that wrote those; entries of one id add
// up.
//
// The roles meet at mbarriers alone: sums_bar when every data warp of the row's CTAs has
// sent its partial sums (to every CTA: a barrier of the whole cluster would also wait for
// the stores under way), ready_bar when a row's entries are prepared, result_bar when its
// sums are known, released_bar when the data warps are done with its entries.  Every wait is
// bounded; one that gives up makes the row's loss and gradient NaN, and the CTA waits no
// more.
//
// The reference of a sum is a whole number n of powers of two: exp(z / tau) is taken as
// 2^n 2^(z log2(e) / tau - n), one fused multiply-add from z, exact in n.  A row whose every
// logit lies below -2^30 powers of two sums to zero against the lowest reference and is done
// again with its maximum subtracted first.
#include <algorithm>

#include "lx_rows.cuh"
#include "lx_tcgen05.cuh"

namespace lx {
namespace {

using namespace rows;

constexpr int SMS = 152;
constexpr int MAX_WARPS = 16;    // data warps of a CTA
constexpr int TEACHERS = 2;      // warps that prepare entries
constexpr int BUFS = 4;          // rows whose entries are held, a multiple of TEACHERS
constexpr int MAX_CLUSTER = 8;
constexpr int SMEM = 222 * 1024; // dynamic shared memory of a CTA at most
constexpr int U = 2;             // pieces of a thread taken together
constexpr int AHEAD = 8;         // pieces asked for before they are used, a multiple of U
constexpr int REGS = 96;         // registers a thread: the launch bound holds the compiler to it
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
  int slice;   // columns of a CTA
  int table;   // places of a table of ids, a power of two
  int rounds;  // pieces of a thread, rounded up to a multiple of U
  int slots;   // of them in shared memory at a time, a multiple of U
  unsigned long long wait_cycles;
  int unmet;   // test hook: the sums' barrier waits for what nobody sends
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
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
// over the lanes of a warp; the same in each
__device__ __forceinline__ void join_warp(float& n, float& s) {
  const float N = warp_max(n);
  s = warp_sum(s * ex2(n - N));
  n = N;
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
__device__ __forceinline__ uint4 pack(const float2* v) {
  if constexpr (sizeof(T) == 4)
    return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y));
  else
    return make_uint4(to_bf2(v[0]), to_bf2(v[1]), to_bf2(v[2]), to_bf2(v[3]));
}
// a piece of -inf, which adds nothing
template <typename T>
__device__ __forceinline__ uint4 no_piece() {
  const uint32_t w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  return make_uint4(w, w, w, w);
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

// Adds U pieces to sums p against reference n.  While the values lie less than 2^40 above
// the reference no maximum is needed; then it is raised to the pieces' maximum.
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

// What a row's sums came to.  `again`: the sums are of the values less `top`.
struct Result {
  float n, s, n1, s1, top;
  bool again;
  __device__ float rel(float z, float ct) const { return again ? (z - top) * ct : fmaf(z, ct, -n); }
  __device__ float rel1(float z) const { return again ? (z - top) * LOG2E : fmaf(z, LOG2E, -n1); }
};

extern __shared__ uint4 distill_smem[];

// TWO: a hard-label term at another temperature than the teacher's.  HELD: rows fit shared
// memory.  blockDim: the data threads and the TEACHERS' warps; gridDim: (CTAs of a row,
// rows)
template <typename T, bool TWO, bool CL, bool HELD>
__global__ void __launch_bounds__(576, 1)
k_distill(const __grid_constant__ DistillArgs A) {
  constexpr int N = Span<T>::N, N2 = N / 2;
  __shared__ float4 red[2][CL ? MAX_CLUSTER : 1][MAX_WARPS];  // the warps' sums
  __shared__ Result res[BUFS];
  __shared__ float msum[BUFS];
  __shared__ int repeats[BUFS];  // whether an id occurs twice
  __shared__ uint64_t sums_bar[2], ready_bar[BUFS], result_bar[BUFS], released_bar[BUFS];
  __shared__ volatile int gave_up;
  const int D = blockDim.x - 32 * TEACHERS, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = D >> 5;
  const bool teacher = warp >= nw;
  const int E1 = A.K + 1, rank = CL ? blockIdx.x : 0, cols = CL ? gridDim.x : 1;
  // entries of BUFS rows: id, z, q, log q; entry K is the label
  int* const eid = (int*)distill_smem;
  float* const ez = (float*)distill_smem + BUFS * E1;
  float* const eq = ez + BUFS * E1;
  float* const elq = eq + BUFS * E1;
  const float ct = A.ct;
  const long first = blockIdx.y, step = gridDim.y;
  auto weight = [&](long t) { return t >= A.T ? 0.f : A.weight ? A.weight[t] : 1.f; };

  auto bar = [](uint64_t* b) { return (uint32_t)__cvta_generic_to_shared(b); };
  if (tid == 0) {
    gave_up = 0;
    for (int i = 0; i < 2; ++i) tcg::mbar_init(bar(&sums_bar[i]), CL ? 1 : nw);
    for (int i = 0; i < BUFS; ++i) {
      tcg::mbar_init(bar(&ready_bar[i]), 1);
      tcg::mbar_init(bar(&result_bar[i]), 1);
      tcg::mbar_init(bar(&released_bar[i]), nw);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if constexpr (CL) cooperative_groups::this_cluster().sync();  // all have started
  bool lost = false;  // a wait of this thread gave up
  auto wait = [&](uint64_t* b, uint32_t parity) {
    if (lost) return;
    if (gave_up || !tcg::mbar_wait(bar(b), parity, &gave_up, A.wait_cycles)) {
      lost = true;
      gave_up = 1;
    }
  };

  if (teacher) {
    // Row k of the CTA's (h, h + TEACHERS, ... are this warp's) has its entries in buffer
    // k % BUFS.
    const int h = warp - nw;
    int* table = (int*)(elq + BUFS * E1) + h * A.table;
    auto prepare = [&](long t, int b) {
      if (weight(t) == 0.f) return;
      int* id = eid + b * E1;
      float *z = ez + b * E1, *q = eq + b * E1, *lq = elq + b * E1;
      const T* row = (const T*)A.logits + t * A.ld;
      for (int i = lane; i < A.table; i += 32) table[i] = -1;
      __syncwarp();
      float tm = -INFINITY;
      bool twice = false;
      for (int j = lane; j < A.K; j += 32) {
        const int e = A.ids[t * A.K + j];
        const bool ok = e >= 0 && e < A.V;
        const float v = ok ? A.top[t * A.K + j] : -INFINITY;
        id[j] = ok ? e : -1;
        z[j] = ok ? to_f32(row[e]) : 0.f;
        q[j] = v;
        tm = fmaxf(tm, v);
        if (ok)  // at least half of the places stay free
          for (int i = e;; ++i) {
            const int was = atomicCAS(&table[i & (A.table - 1)], -1, e);
            twice |= was == e;
            if (was == -1 || was == e) break;
          }
      }
      twice = __any_sync(0xffffffffu, twice);
      if (lane == 0) {
        const int e = A.labels ? A.labels[t] : -1;
        const bool ok = e >= 0 && e < A.V;
        id[A.K] = ok ? e : -1;
        z[A.K] = ok ? to_f32(row[e]) : 0.f;
        q[A.K] = 0.f;
        repeats[b] = twice;
      }
      tm = warp_max(tm);
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
      if (lane == 0) msum[b] = m;
    };
    auto provide = [&](long k) {
      const long t = first + k * step;
      if (t >= A.T) return;
      if (k >= BUFS) wait(&released_bar[k % BUFS], (uint32_t)(k / BUFS - 1) & 1);
      if (!__any_sync(0xffffffffu, lost)) prepare(t, (int)(k % BUFS));
      __syncwarp();
      if (lane == 0) tcg::mbar_arrive(bar(&ready_bar[k % BUFS]));
    };
    for (long k = h; k < BUFS; k += TEACHERS) provide(k);
    for (long k = h; first + k * step < A.T; k += TEACHERS) {
      const long t = first + k * step;
      const int b = (int)(k % BUFS);
      wait(&result_bar[b], (uint32_t)(k / BUFS) & 1);
      const float w = weight(t);
      const Result r = res[b];
      const int* id = eid + b * E1;
      const float *zj = ez + b * E1, *q = eq + b * E1, *lq = elq + b * E1;
      float loss = 0.f;
      if (w != 0.f && r.s != 0.f) {
        const float ls = logf(r.s);
        for (int j = lane; j < A.K; j += 32)
          if (q[j] != 0.f) loss += q[j] * (lq[j] - (r.rel(zj[j], ct) * LN2 - ls));
        loss = warp_sum(loss) * A.a * A.tau * A.tau;
        if (A.b != 0.f && id[A.K] >= 0)
          loss += A.b * (logf(r.s1) - (TWO ? r.rel1(zj[A.K]) : r.rel(zj[A.K], ct)) * LN2);
        loss *= w;
      }
      if (__any_sync(0xffffffffu, lost)) loss = NAN;
      if (lane == 0 && rank == 0) A.loss[t] = loss;
      __syncwarp();
      provide(k + BUFS);
    }
  } else {
    const int v0 = rank * A.slice, vn = min(A.slice, A.V - v0);
    const char* const slot = (const char*)(distill_smem + (4 * BUFS * E1 + TEACHERS * A.table + 3) / 4 + tid);
    const uint32_t slot_at = (uint32_t)__cvta_generic_to_shared(slot);
    const uint32_t apart = D * 16, batch = U * apart, ring = A.slots * apart;  // bytes between a thread's pieces
    auto advance = [&](uint32_t& k) { k = k + batch == ring ? 0 : k + batch; };
    auto span = [&](long t) { return Span<T>((const T*)A.logits + (t < A.T ? t : first) * A.ld + v0, vn); };
    auto pieces_of = [&](const Span<T>& S) { return (S.pieces - tid + D - 1) / D; };  // of this thread

    // The copies, a batch to a group, in the order of use: rows of weight 0 and pieces that
    // a thread does not have leave their slots as they are.
    long ask_t = first;
    float ask_w = weight(first);
    const T* ask_at = nullptr;
    int ask_left = 0, ask_rounds = 0;  // pieces of the thread, rounds of the row not asked for yet
    auto ask = [&](uint32_t to) {
      if (ask_rounds == 0) {
        const Span<T> S = span(ask_t);
        ask_at = S.piece(tid);
        ask_left = ask_w != 0.f ? pieces_of(S) : 0;
        ask_rounds = A.rounds;
        ask_t += step;
        ask_w = weight(ask_t);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u < ask_left)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slot_at + to + u * apart),
                       "l"(ask_at + (long)u * D * N)
                       : "memory");
      asm volatile("cp.async.commit_group;" ::: "memory");
      ask_at += (long)U * D * N;
      ask_left -= U;
      ask_rounds -= U;
    };
    auto landed = [] { asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD / U) : "memory"); };

    // The first pass: a batch of the thread's pieces, of which it has `have`, into the sums
    auto take = [&](Run& r, const uint4* q) {
      add_pieces<T>(r.n, r.p, q, ct);
      if (TWO) add_pieces<T>(r.n1, r.p1, q, LOG2E);
    };
    auto take_edge = [&](Run& r, float v) {
      add_value(r.n, r.p, v, ct);
      if (TWO) add_value(r.n1, r.p1, v, LOG2E);
    };
    auto take_slots = [&](Run& r, uint32_t k, int have) {
      uint4 q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u] = u < have ? *(const uint4*)(slot + k + u * apart) : no_piece<T>();
      take(r, q);
    };
    uint32_t k0 = 0, k1 = 0, k2 = 0;  // slots of the copies, of the first and of the second pass
    // of a whole row by itself: the first row, and every row where there is no gradient
    auto pass1 = [&](const Span<T>& S, float w, Run& r) {
      const int n = w != 0.f ? pieces_of(S) : 0;
      if constexpr (HELD) {
        for (int p = 0; p < A.rounds; p += U) {
          ask(k0);
          advance(k0);
          landed();
          if (p < n) take_slots(r, k1, n - p);
          advance(k1);
        }
      } else {
        for (int p = 0; p < n; p += U) {
          uint4 q[U];
#pragma unroll
          for (int u = 0; u < U; ++u)
            q[u] = p + u < n ? *(const uint4*)S.piece((p + u) * D + tid) : no_piece<T>();
          take(r, q);
        }
      }
      if (w != 0.f && tid < S.edges) take_edge(r, to_f32(S.row[S.edge(tid)]));
    };

    // Every data warp's v of the row's CTAs, in red[]; returns which half
    int sent = 0;
    auto exchange = [&](float4 v) {
      const int turn = sent & 1;
      if (__any_sync(0xffffffffu, lost)) return turn;
      if constexpr (CL) {
        if (tid == 0) tcg::mbar_expect_tx(bar(&sums_bar[turn]), cols * nw * 16 + (A.unmet ? 16 : 0));
        if (lane < cols) {
          uint32_t to, at;
          asm("mapa.shared::cluster.u32 %0, %1, %2;"
              : "=r"(to)
              : "r"((uint32_t)__cvta_generic_to_shared(&red[turn][rank][warp])), "r"(lane));
          asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(bar(&sums_bar[turn])), "r"(lane));
          asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(
                           to),
                       "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(at)
                       : "memory");
        }
      } else if (lane == 0) {
        red[turn][0][warp] = v;
        if (!(A.unmet && warp == 0)) tcg::mbar_arrive(bar(&sums_bar[turn]));
      }
      __syncwarp();
      wait(&sums_bar[turn], (sent >> 1) & 1);
      ++sent;
      return turn;
    };
    // The threads' sums over the row, the same in every data thread
    auto joined = [&](Run r) {
      r.s += r.p.x + r.p.y;
      join_warp(r.n, r.s);
      if (TWO) {
        r.s1 += r.p1.x + r.p1.y;
        join_warp(r.n1, r.s1);
      }
      const int turn = exchange(make_float4(r.n, r.s, r.n1, r.s1));
      r = Run();
      for (int i = lane; i < cols * MAX_WARPS; i += 32)
        if ((i & (MAX_WARPS - 1)) < nw) {
          const float4 o = red[turn][i / MAX_WARPS][i & (MAX_WARPS - 1)];
          join(r.n, r.s, o.x, o.y);
          if (TWO) join(r.n1, r.s1, o.z, o.w);
        }
      join_warp(r.n, r.s);
      if (TWO) join_warp(r.n1, r.s1);
      if (__any_sync(0xffffffffu, lost)) r.s = r.s1 = NAN;
      return r;
    };

    float w = weight(first), wn = weight(first + step);
    Run run;  // the sums of row t
    if constexpr (HELD)
      for (int p = 0; p < AHEAD; p += U) {
        ask(k0);
        advance(k0);
      }
    pass1(span(first), w, run);
    long k = 0;  // the CTA's rows
    for (long t = first; t < A.T; t += step, ++k) {
      const Span<T> S = span(t), Sn = span(t + step);
      const float wn2 = weight(t + 2 * step);
      const int b = (int)(k % BUFS);
      bool dead = w == 0.f;  // nothing to learn
      Result r = {0.f, 0.f, 0.f, 0.f, 0.f, false};
      wait(&ready_bar[b], (uint32_t)(k / BUFS) & 1);
      if (!dead) {
        run = joined(run);
        if (run.s == 0.f) {  // every logit is -inf or out of the references' reach
          r.again = true;
          float top = -INFINITY;
          for (int i = tid; i < S.pieces; i += D) top = fmaxf(top, piece_max<T>(*(const uint4*)S.piece(i)));
          if (tid < S.edges) top = fmaxf(top, to_f32(S.row[S.edge(tid)]));
          const int turn = exchange(make_float4(warp_max(top), 0.f, 0.f, 0.f));
          top = -INFINITY;
          for (int i = lane; i < cols * MAX_WARPS; i += 32)
            if ((i & (MAX_WARPS - 1)) < nw) top = fmaxf(top, red[turn][i / MAX_WARPS][i & (MAX_WARPS - 1)].x);
          r.top = top = warp_max(top);
          dead = top == -INFINITY;
          if (!dead) {
            run = Run();
            run.n = run.n1 = 0.f;
            auto add = [&](float v) {
              run.s += ex2((v - top) * ct);
              if (TWO) run.s1 += ex2((v - top) * LOG2E);
            };
            for (int i = tid; i < S.pieces * N; i += D) add(to_f32(S.row[S.head + i]));
            if (tid < S.edges) add(to_f32(S.row[S.edge(tid)]));
            run = joined(run);
          }
        }
        r.n = run.n;
        r.s = dead ? 0.f : run.s;
        r.n1 = TWO ? run.n1 : run.n;
        r.s1 = TWO ? run.s1 : run.s;
      }
      if (tid == 0) {
        res[b] = r;
        tcg::mbar_arrive(bar(&result_bar[b]));
      }
      Run next;  // the sums of row t + step
      if (!A.dlogits) {
        if (t + step < A.T) pass1(Sn, wn, next);
      } else {
        const int* id = eid + b * E1;
        const float *zj = ez + b * E1, *q = eq + b * E1;
        T* dz = (T*)A.dlogits + t * A.ldd + v0;
        const bool same = (((uintptr_t)dz ^ (uintptr_t)S.row) & 15) == 0;
        const int label = dead ? -1 : id[A.K];
        const float qa = dead ? 0.f : w * A.a * A.tau, hb = label < 0 ? 0.f : w * A.b;
        const float pb = dead ? 0.f : hb / r.s1, pa = dead ? 0.f : qa * msum[b] / r.s + (TWO ? 0.f : pb);
        auto value = [&](float z) {
          if (dead) return 0.f;
          return TWO ? pa * ex2(r.rel(z, ct)) + pb * ex2(r.rel1(z)) : pa * ex2(r.rel(z, ct));
        };
        const float2 pa2 = both(pa), pb2 = both(pb), neg = both(-r.n), neg1 = both(-r.n1);
        auto gradient = [&](uint4 x4) {
          float2 v[N2];
          unpack<T>(x4, v);
#pragma unroll
          for (int j = 0; j < N2; ++j) {
            const float2 x = fma2(v[j], both(ct), neg);
            float2 o = mul2(make_float2(ex2(x.x), ex2(x.y)), pa2);
            if (TWO) {
              const float2 x1 = fma2(v[j], both(LOG2E), neg1);
              o = fma2(make_float2(ex2(x1.x), ex2(x1.y)), pb2, o);
            }
            v[j] = o;
          }
          return pack<T>(v);
        };
        // a piece of a row that is dead or done again, or whose gradient starts elsewhere
        // within 16 bytes
        auto odd_piece = [&](const uint4* from, T* out) {
          uint4 x = make_uint4(0u, 0u, 0u, 0u);
          if (!dead) {
            x = *from;
            if (r.again) {
              float2 v[N2];
              unpack<T>(x, v);
#pragma unroll
              for (int j = 0; j < N2; ++j) v[j] = make_float2(value(v[j].x), value(v[j].y));
              x = pack<T>(v);
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
        const int n = pieces_of(S), n_next = wn != 0.f ? pieces_of(Sn) : 0;
        const bool plain = same && !r.again && !dead;
        if constexpr (HELD) {
          const float edge = wn != 0.f && tid < Sn.edges ? to_f32(Sn.row[Sn.edge(tid)]) : 0.f;
          // the thread's batches that are whole in both rows, then the others
          const int full = plain ? min(n, n_next) / U * U : 0;
          int p = 0;
          for (; p < full; p += U) {
            uint4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = *(const uint4*)(slot + k2 + u * apart);
#pragma unroll
            for (int u = 0; u < U; ++u) *(uint4*)(out + (long)u * D * N) = gradient(x[u]);
            ask(k2);  // the values have been used: the places are free
            advance(k2);
            landed();
            take_slots(next, k1, U);
            advance(k1);
            out += (long)U * D * N;
          }
          for (; p < A.rounds; p += U) {
            for (int u = 0; u < U && p + u < n; ++u)
              odd_piece((const uint4*)(slot + k2 + u * apart), out + (long)u * D * N);
            ask(k2);
            advance(k2);
            landed();
            if (p < n_next) take_slots(next, k1, n_next - p);
            advance(k1);
            out += (long)U * D * N;
          }
          if (wn != 0.f && tid < Sn.edges) take_edge(next, edge);
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
            float x = q[j];
            if (repeats[b] || id[j] == label) {  // (the label may be one of the entries)
              x = 0.f;
              for (int i = 0; i < A.K; ++i) x += id[i] == id[j] ? q[i] : 0.f;
            }
            dz[e] = from_f32<T>(value(zj[j]) - qa * x - (id[j] == label ? hb : 0.f));
          }
        if constexpr (!HELD)
          if (t + step < A.T) pass1(Sn, wn, next);
      }
      __syncwarp();
      if (lane == 0) tcg::mbar_arrive(bar(&released_bar[b]));
      run = next;
      w = wn;
      wn = wn2;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  }
  if constexpr (CL) {
    // A CTA's shared memory outlives what its neighbours send; after a wait that gave up
    // that may still be on its way: some ten microseconds for it.
    if (gave_up)
      for (const long long c0 = clock64(); clock64() - c0 < 20000;) {}
    cooperative_groups::this_cluster().sync();
  }
}

template <typename T, bool TWO, bool CL, bool HELD>
lx_status launch_distill(const DistillArgs& A, int threads, int cols, int groups, size_t smem, cudaStream_t s) {
  static bool cap[64] = {};
  int dev = 0;
  LX_CUDA(cudaGetDevice(&dev));
  LX_CUDA(smem_cap_once((const void*)k_distill<T, TWO, CL, HELD>, SMEM, dev, cap));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cols, groups);
  cfg.blockDim = dim3(threads + 32 * TEACHERS);
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
  const CallWaits waits = take_call_waits();
  A.wait_cycles = waits.cycles;
  A.unmet = waits.unmet == LX_WAIT_CALL_SUMS;
  // Data threads that hold `bytes` of a row, and the CTAs of a row: as many as it takes to
  // hold it, and more where rows are few, in slices of 4096 columns at least
  A.table = 32;
  while (A.table < 2 * K) A.table *= 2;
  const size_t entries = ((4 * BUFS * (size_t)(K + 1) + TEACHERS * A.table + 3) / 4) * 16;
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
  const int ctas = std::max(1, std::min((int)(65536 / (REGS * (threads + 32 * TEACHERS))), (int)(227 * 1024 / (smem + 5120))));
  const int groups = std::min(T, std::max(1, SMS * ctas / cols));
  const bool two = ce_weight != 0.f && temperature != 1.f;
  cudaStream_t s = (cudaStream_t)stream;
  return dtype == LX_BF16 ? launch_type<__nv_bfloat16>(A, two, threads, cols, groups, smem, s)
                          : launch_type<float>(A, two, threads, cols, groups, smem, s);
}
