// Distillation from a teacher's stored top logits (lx_distill_loss).  For a token
// with student logits z [V], teacher entries (id_j, t_j), weight w:
//   q_j = softmax_j(t_j / tau) over the valid entries, or exp(t_j / tau - L),
//   kd  = sum_j q_j (log q_j - log p_{id_j}),  p = softmax(z / tau),  m = sum_j q_j
//   ce  = log sum_v exp z_v - z_label
//   loss = w (a tau^2 kd + b ce)
//   dz_v = w (a tau (m p_v - sum_{j: id_j = v} q_j) + b (softmax(z)_v - [v = label])).
//
// Bound by the logits: they are read from memory once and their gradient is written
// once.  Short rows are held in registers (k_distill_short).  For the others a CTA (or a
// cluster of CTAs, where a row is long or rows are few) works on one row at a time.  Its
// threads hold their part of the row as 16-byte pieces in shared memory, each thread its own
// (cp.async, no barrier between copy and use).  The first pass over a row sums the
// exponentials against a running reference, an exchange joins the sums, the second pass
// writes the gradient.  The passes run together, the first a row and `lead` pieces before
// the second: a thread finishes a batch of pieces, asks for later ones in their place, and
// takes the first pass's next batch, which was asked for AHEAD pieces ago.  So reads and
// writes go on all the time (with the passes one after the other all CTAs drew on memory in
// the same halves of their rows), and a row's sums are on their way while the second pass
// finishes the row before.  Rows that do not fit the shared memory of eight CTAs are read a
// second time from L2.
//
// Two to four warps of their own prepare the teacher's entries, up to four rows ahead (their
// chains of loads take longer than a row), write the losses and, once the dense values of a
// row are written, the entries' places once more; entries of one id add up.
//
// The roles meet at mbarriers alone: sums_bar when every data warp of the row's CTAs has
// sent its partial sums (to every CTA: a barrier of the whole cluster would also wait for
// the stores under way), ready_bar when a row's entries are prepared, result_bar when its
// sums are known, released_bar when the data warps have written it.  Every wait is
// bounded.  After one that gives up its CTA waits no more and runs to its end, where the
// rows that were not done by then are made NaN, in all of their CTAs.
//
// The reference of a sum is a whole number n of powers of two: exp(z / tau) is taken as
// 2^n 2^(z log2(e) / tau - n), one fused multiply-add from z, exact in n.  A row whose
// largest logit lies some 2^30 powers of two from zero or further, where n is off by its own
// rounding, sums to zero or infinity and is done again with its maximum subtracted first.
#include <cooperative_groups.h>

#include <algorithm>
#include <type_traits>

#include "lx_rows.cuh"
#include "lx_tcgen05.cuh"

namespace lx {
namespace {

using namespace rows;

constexpr int MAX_WARPS = 16;    // data warps of a CTA
constexpr int BUFS = 4;          // rows whose entries are held
constexpr int MAX_TEACHERS = 4;  // warps that prepare entries: 2, or 4 beside 16 data warps
constexpr int MAX_CLUSTER = 8;
constexpr int SMEM = 218880;     // dynamic shared memory of an SM's CTAs at most
constexpr int U = 2;             // pieces of a thread taken together
// pieces asked for before they are used, a multiple of U: rows held for a gradient leave
// less room
constexpr int ahead_of(bool grad) { return grad ? 6 : 12; }
constexpr int LEAD = 4;          // of the first pass, a multiple of U (or a row, if that is less)
constexpr int SENDS = 4;         // exchanges whose sums are held
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
  int log_d;   // log2 of a CTA's data threads
  int teachers;
  int table;   // places of a table of ids, a power of two
  int rounds;  // pieces of a thread, rounded up to a multiple of U
  int slots;   // of them in shared memory at a time, a multiple of U
  int lead;
  unsigned long long wait_cycles;
  // test hook: barriers that nobody tells of what they wait for
  int sums_met;                       // exchanges that are told of, SENDS + 2 for all
  unsigned entries_met, written_met;  // a CTA's rows whose entries, whose dense gradient are told of
};

__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
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
        const float2 x = fmas(v[j], both(c), both(neg));
        s = adds(s, make_float2(ex2(x.x), ex2(x.y)));
      }
    }
    return s;
  };
  float2 s;
  if (n == LOWEST || (s = sum(-n), fmaxf(s.x, s.y) > 1099511627776.f)) {  // (a NaN goes on as it is)
    float mx = piece_max<T>(q[0]);
    for (int u = 1; u < U; ++u) mx = fmaxf(mx, piece_max<T>(q[u]));
    const float N = fmaxf(LOWEST, ceilf(mx * c));
    p = muls(p, both(ex2(n - N)));
    n = N;
    s = sum(-n);
  }
  p = adds(p, s);
}
__device__ __forceinline__ void add_value(float& n, float2& p, float v, float c) {
  const float t = v * c;
  if (t > n + 16.f) {
    const float N = ceilf(t);
    p = muls(p, both(ex2(n - N)));
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

// A row's gradient is pa 2^rel + pb 2^rel1 (one term without a second temperature), less
// qa q at an entry and hb at the label
struct Factors {
  float qa, hb, pa, pb;
  __device__ float value(const Result& r, float z, float ct, bool two) const {
    return two ? pa * ex2(r.rel(z, ct)) + pb * ex2(r.rel1(z)) : pa * ex2(r.rel(z, ct));
  }
};
__device__ __forceinline__ Factors factors(const DistillArgs& A, const Result& r, float w, float m, int label, bool two) {
  Factors f;
  f.qa = w * A.a * A.tau;
  f.hb = label < 0 ? 0.f : w * A.b;
  f.pb = f.hb / r.s1;
  f.pa = f.qa * m / r.s + (two ? 0.f : f.pb);
  return f;
}

// The gradient of a piece.  bf16: the factors go into the exponents (a 2^x = 2^(x + log2 a),
// which rounds to 5e-5 of the value at most while the reference is below 2^10, a fortieth of
// what the bf16 rounds to); fp32: multiplied.
template <typename T, bool TWO>
struct Gradient {
  static constexpr int N2 = 8 / sizeof(T);
  static constexpr bool FOLD = sizeof(T) == 2;
  float ct;
  float2 pa2, pb2, neg, neg1;
  __device__ Gradient(const DistillArgs& A, const Result& r, const Factors& f)
      : ct(A.ct),
        pa2(both(f.pa)),
        pb2(both(f.pb)),
        neg(both((FOLD ? lg2(f.pa) : 0.f) - r.n)),
        neg1(both((FOLD ? lg2(f.pb) : 0.f) - r.n1)) {}
  // whether it does not hold: negative factors, references that would swallow the factors,
  // and a maximum that was subtracted
  __device__ static bool slow(const Result& r, const Factors& f) {
    return r.again || (FOLD && (f.pa < 0.f || f.pb < 0.f || fmaxf(fabsf(r.n), TWO ? fabsf(r.n1) : 0.f) > 1024.f));
  }
  __device__ uint4 operator()(uint4 x4) const {
    float2 v[N2];
    unpack<T>(x4, v);
#pragma unroll
    for (int j = 0; j < N2; ++j) {
      const float2 x = fmas(v[j], both(ct), neg);
      float2 o = make_float2(ex2(x.x), ex2(x.y));
      if (!FOLD) o = muls(o, pa2);
      if (TWO) {
        const float2 x1 = fmas(v[j], both(LOG2E), neg1), o1 = make_float2(ex2(x1.x), ex2(x1.y));
        o = FOLD ? adds(o, o1) : fmas(o1, pb2, o);
      }
      v[j] = o;
    }
    return pack<T>(v);
  }
};

// A table of a row's ids: open addressing, a free place is -1 and at least half of the places
// are; an id e that was put in more than once is kept as -2 - e.
__device__ __forceinline__ bool put_id(int* table, int size, int e) {  // whether it was there
  for (unsigned i = e;; ++i) {
    int* const at = table + (i & (size - 1));
    const int was = atomicCAS(at, -1, e);
    if (was == -1) return false;
    if (was == e || was == -2 - e) {
      *(volatile int*)at = -2 - e;
      return true;
    }
  }
}
__device__ __forceinline__ int times_of(const int* table, int size, int e) {  // 0, 1, or 2 for more
  for (unsigned i = e;; ++i) {
    const int was = table[i & (size - 1)];
    if (was == -1) return 0;
    if (was == e) return 1;
    if (was == -2 - e) return 2;
  }
}
// What the entries of id[j], entry j's, add up to, in their order; -1 where entry K, the label,
// has its place written by another entry.  Only ids that are repeated are added up: a store
// of top logits has few (5072 rows of 16384 bf16, 56 entries: 74 us, 78 where a repeat sent
// all of its row's entries here; 1000 random ids, an eighth of them repeats: 1428 and 1005 us
// at 4096 columns).
__device__ __forceinline__ float entries_of(const int* id, const float* q, int K, int j, bool twice, const int* table,
                                            int size) {
  const int e = id[j];
  if (!twice && j < K) return q[j];
  const int times = times_of(table, size, e);
  if (j == K) return times == 0 ? 0.f : -1.f;
  if (times == 1) return q[j];
  float x = 0.f;
  for (int i = 0; i < K; ++i) x += id[i] == e ? q[i] : 0.f;
  return x;
}

// Waits, after a wait that gave up, until all that was sent to a barrier of this CTA has landed.
// `sent` counts the 16-byte sums that a CTA's warps sent to each CTA (in every CTA), `told` the rows
// that the barrier was told to expect, `each` sums a row.  At most one phase is open: a warp
// sends for row x + 4 after it received row x + 2, for which every warp had sent, each after
// it received row x, the barrier's last.  The open phase's account is brought to what was
// sent, so that it ends with the last byte.
__device__ __forceinline__ void await_sent(uint32_t bar, unsigned* sent, unsigned told, int each, int cols,
                                           unsigned long long cycles) {
  unsigned sums = 0;
#pragma unroll 1
  for (int c = 0; c < cols; ++c) sums += *cooperative_groups::this_cluster().map_shared_rank(sent, c);
  const int more = (int)(sums - told * each);  // sent, less expected
  if (more < 0)
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(-16 * more) : "memory");
  if (more > 0) {
    tcg::mbar_expect_tx(bar, 16 * more);
    ++told;
  }
  const long long c0 = clock64();  // (a barrier of no rows counts as past its phase 1)
  while (!tcg::mbar_try_wait(bar, (told - 1) & 1) && clock64() - c0 < (long long)cycles) {}
}

// What a wait that gave up left of the CTA's rows (first, first + step, ...): row k's gradient, and
// its loss unless NULL, become NaN from lost[k % teachers] on, rows of weight 0 apart, which
// wait for nothing.  (Inlined, as a call's registers cost the rows before 3 %.)
template <typename T>
__device__ __forceinline__ void rows_lost(const unsigned* lost, int teachers, unsigned first, unsigned step, unsigned T0,
                                          const float* weight, float* loss, T* dz, long ldd, int vn) {
#pragma unroll 1
  for (unsigned k = 0, t = first; t < T0; ++k, t += step) {
    if (k < lost[k % teachers] || (weight && weight[t] == 0.f)) continue;
    if (loss && threadIdx.x == 0) loss[t] = NAN;
#pragma unroll 1
    for (int e = threadIdx.x; e < vn; e += blockDim.x) dz[(long)t * ldd + e] = from_f32<T>(NAN);
  }
}

extern __shared__ uint4 distill_smem[];

// TWO: a hard-label term at another temperature than the teacher's.  HELD: rows fit shared
// memory.  blockDim: the data threads and the teachers' warps; gridDim: (CTAs of a row,
// rows)
template <typename T, bool TWO, bool CL, bool HELD, bool GRAD>
__global__ void __launch_bounds__(640, 1)
k_distill(const __grid_constant__ DistillArgs A) {
  constexpr int N = Span<T>::N, N2 = N / 2, AHEAD = ahead_of(GRAD);
  // the warps' sums of SENDS rows, and of a row that is done again
  __shared__ float4 red[SENDS + 2][CL ? MAX_CLUSTER : 1][MAX_WARPS];
  __shared__ Result res[BUFS];
  __shared__ struct {
    Result r;
    Factors f;
  } own[MAX_WARPS];  // a data warp's copy for its odd pieces, which keep no registers
  __shared__ float msum[BUFS];
  __shared__ uint64_t sums_bar[SENDS + 2], ready_bar[BUFS], result_bar[BUFS], released_bar[BUFS];
  __shared__ unsigned sent[CL ? SENDS + 2 : 1], told[CL ? SENDS + 2 : 1];  // of await_sent, by barrier
  __shared__ volatile int gave_up;  // a wait of the CTA did
  __shared__ unsigned lost_from[MAX_TEACHERS];  // a teacher's first row that was not done then, in any CTA
  const int log_d = A.log_d, D = 1 << log_d, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = D >> 5;
  const bool teacher = warp >= nw;
  const int E1 = A.K + 1, rank = CL ? blockIdx.x : 0, cols = CL ? gridDim.x : 1;
  // entries of BUFS rows: id, z, q, log q; entry K is the label
  int* const eid = (int*)distill_smem;
  float* const ez = (float*)distill_smem + BUFS * E1;
  float* const eq = ez + BUFS * E1;
  float* const elq = eq + BUFS * E1;
  const float ct = A.ct;
  const unsigned T0 = A.T, first = blockIdx.y, step = gridDim.y;  // (row + 3 * step stays below 2^32)
  auto weight = [&](unsigned t) { return t >= T0 ? 0.f : A.weight ? A.weight[t] : 1.f; };

  auto bar = [](uint64_t* b) { return (uint32_t)__cvta_generic_to_shared(b); };
  if (tid == 0) {
    gave_up = 0;
    for (int i = 0; i < MAX_TEACHERS; ++i) lost_from[i] = ~0u;
    for (int i = 0; i < SENDS + 2; ++i) {
      tcg::mbar_init(bar(&sums_bar[i]), CL ? 1 : nw);
      if (CL) sent[i] = told[i] = 0;
    }
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
    if (lost || (!gave_up && tcg::mbar_try_wait(bar(b), parity))) return;
    const long long c0 = clock64();
    while (!gave_up && clock64() - c0 < (long long)A.wait_cycles) {
      if (teacher) __nanosleep(200);  // its polls would take the data warps' issue slots
      if (tcg::mbar_try_wait(bar(b), parity)) return;
    }
    lost = true;
    gave_up = 1;
  };

  if (teacher) {
    // Row k of the CTA's (h, h + A.teachers, ... are this warp's) has its entries in buffer
    // k % BUFS.
    const int h = warp - nw;
    int* table = (int*)(elq + BUFS * E1) + h * A.table;
    unsigned lost_k = ~0u;  // the first row that was not done when a wait gave up
    auto prepare = [&](unsigned t, int b) {
      int* id = eid + b * E1;
      float *z = ez + b * E1, *q = eq + b * E1, *lq = elq + b * E1;
      const T* row = (const T*)A.logits + (long)t * A.ld;
      const float w = weight(t), stored = A.top_lse ? A.top_lse[t] : 0.f;
      const int label = A.labels ? A.labels[t] : -1;
      float tm = -INFINITY;
      for (int j = lane; j < A.K; j += 32) {
        const int e = A.ids[(long)t * A.K + j];
        const float v = A.top[(long)t * A.K + j];
        const bool ok = e >= 0 && e < A.V && v != -INFINITY;  // (a store's padding may hold any id)
        id[j] = ok ? e : -1;
        q[j] = ok ? v : -INFINITY;
        tm = fmaxf(tm, q[j]);
      }
      if (w == 0.f) return;
      for (int j = lane; j < A.K; j += 32) z[j] = id[j] >= 0 ? to_f32(row[id[j]]) : 0.f;
      if (lane == 0) {
        const bool ok = label >= 0 && label < A.V;
        id[A.K] = ok ? label : -1;
        z[A.K] = ok ? to_f32(row[label]) : 0.f;
        q[A.K] = 0.f;
      }
      tm = warp_max(tm);
      float lz;  // log of the distribution's sum, relative to tm / tau
      if (A.top_lse) {
        lz = stored - tm / A.tau;
      } else {
        float s = 0.f;
        for (int j = lane; j < A.K; j += 32)
          if (id[j] >= 0) s += expf((q[j] - tm) / A.tau);
        lz = logf(warp_sum(s));
      }
      float m = 0.f;
      for (int j = lane; j < A.K; j += 32) {
        const float l = id[j] >= 0 ? (q[j] - tm) / A.tau - lz : -INFINITY;
        const float p = expf(l);
        lq[j] = l;
        q[j] = p;
        m += p;
      }
      m = warp_sum(m);
      if (lane == 0) msum[b] = m;
    };
    auto provide = [&](unsigned k, unsigned t) {
      if (t >= T0) return;
      if (!__any_sync(0xffffffffu, lost)) prepare(t, k % BUFS);
      __syncwarp();
      if (lane == 0 && k < A.entries_met) tcg::mbar_arrive(bar(&ready_bar[k % BUFS]));
    };
    // fills the table; whether an id of the row occurs twice
    auto repeated = [&](const int* id) {
      for (int i = lane; i < A.table; i += 32) table[i] = -1;
      __syncwarp();
      bool twice = false;
      for (int j = lane; j < A.K; j += 32)
        if (id[j] >= 0) twice |= put_id(table, A.table, id[j]);
      twice = __any_sync(0xffffffffu, twice);
      __syncwarp();  // the table may be read
      return twice;
    };
    for (unsigned k = h; k < BUFS; k += A.teachers) provide(k, first + k * step);
    unsigned t = first + h * step;
    for (unsigned k = h; t < T0; k += A.teachers, t += A.teachers * step) {
      const int b = k % BUFS;
      const uint32_t parity = k / BUFS & 1;
      wait(&result_bar[b], parity);
      const float w = weight(t);
      const Result r = res[b];
      const int* id = eid + b * E1;
      const float *zj = ez + b * E1, *q = eq + b * E1, *lq = elq + b * E1;
      const bool dead = w == 0.f || r.s == 0.f;
      float loss = 0.f;
      if (!dead) {
        const float ls = logf(r.s);
        for (int j = lane; j < A.K; j += 32)
          if (q[j] != 0.f) loss += q[j] * (lq[j] - (r.rel(zj[j], ct) * LN2 - ls));
        loss = warp_sum(loss) * A.a * A.tau * A.tau;
        if (A.b != 0.f && id[A.K] >= 0)
          loss += A.b * (logf(r.s1) - (TWO ? r.rel1(zj[A.K]) : r.rel(zj[A.K], ct)) * LN2);
        loss *= w;
      }
      if (!GRAD && w != 0.f && __any_sync(0xffffffffu, lost || gave_up)) loss = NAN;  // (rows_lost does it else)
      if (lane == 0 && rank == 0) A.loss[t] = loss;
      const bool twice = GRAD && !dead && repeated(id);
      wait(&released_bar[b], parity);
      // A row is done once its dense values lie there and nothing gave up before, in any of its
      // CTAs; else all of it is written anew at the end.
      const bool done = !__any_sync(0xffffffffu, lost || gave_up);
      if (!done) lost_k = min(lost_k, k);
      if (GRAD && !dead && done) {
        // the entries of this CTA's columns; the label may be one of them
        T* dz = (T*)A.dlogits + (long)t * A.ldd;
        const int label = id[A.K], v0 = rank * A.slice, vn = min(A.slice, A.V - v0);
        const Factors f = factors(A, r, w, msum[b], label, TWO);
        for (int j = lane; j <= A.K; j += 32) {
          const int e = id[j];
          if (e < v0 || e >= v0 + vn) continue;
          const float x = entries_of(id, q, A.K, j, twice, table, A.table);
          if (x == -1.f) continue;
          dz[e] = from_f32<T>(f.value(r, zj[j], ct, TWO) - f.qa * x - (e == label ? f.hb : 0.f));
        }
      }
      __syncwarp();
      provide(k + BUFS, t + BUFS * step);
    }
    if (lane == 0 && lost_k != ~0u) {
      if constexpr (CL)
#pragma unroll 1
        for (int c = 0; c < cols; ++c)
          atomicMin(cooperative_groups::this_cluster().map_shared_rank(&lost_from[h], c), lost_k);
      else lost_from[h] = lost_k;
    }
  } else {
    const int v0 = rank * A.slice, vn = min(A.slice, A.V - v0);
    const uint32_t slot = (uint32_t)__cvta_generic_to_shared(distill_smem + (4 * BUFS * E1 + A.teachers * A.table + 3) / 4 + tid);
    auto from_slot = [](uint32_t at) {
      uint4 q;
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(at) : "memory");
      return q;
    };
    const uint32_t apart = D * 16, batch = U * apart, ring = A.slots * apart;  // bytes between a thread's pieces
    auto advance = [&](uint32_t& k) { k = k + batch == ring ? 0 : k + batch; };
    auto span = [&](unsigned t) { return Span<T>((const T*)A.logits + (long)(t < T0 ? t : first) * A.ld + v0, vn); };
    auto pieces_of = [&](const Span<T>& S) { return (S.pieces - tid + D - 1) >> log_d; };  // of this thread
    auto whole_of = [&](const Span<T>& S) { return (S.pieces - (tid | 31) + D - 1) >> log_d; };  // of each of its warp's

    // The copies, a batch to a group, in the order of use: rows of weight 0 and pieces that
    // a thread does not have leave their slots as they are.
    unsigned ask_t = first;
    float ask_w = weight(first);
    const T* ask_at = nullptr;
    // not asked for yet: pieces of the thread, pieces that every thread has, rounds of the row
    int ask_left = 0, ask_whole = 0, ask_rounds = 0;
    auto copy = [](uint32_t dst, const void* src) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    };
    auto ask_row = [&] {
      if (ask_rounds == 0) {
        const Span<T> S = span(ask_t);
        ask_at = S.piece(tid);
        ask_left = ask_w != 0.f ? pieces_of(S) : 0;
        ask_whole = ask_w != 0.f ? whole_of(S) : 0;
        ask_rounds = A.rounds;
        ask_t += step;
        ask_w = weight(ask_t);
      }
    };
    auto ask = [&](uint32_t to) {
      ask_row();
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u < ask_left) copy(slot + to + u * apart, ask_at + (long)u * D * N);
      asm volatile("cp.async.commit_group;" ::: "memory");
      ask_at += (long)U * D * N;
      ask_left -= U;
      ask_whole -= U;
      ask_rounds -= U;
    };
    int feed_sent = 0;  // rows whose sums this warp sent
    // Sums of the row's CTAs: every data warp's v goes to red[i] of each of them.  A warp that gave
    // up sends no more.
    auto send = [&](int i, float4 v) {
      if (__any_sync(0xffffffffu, lost)) {
        --feed_sent;  // (of a row that is done again, nothing is sent then)
        return;
      }
      if constexpr (CL) {
        if (tid == 0 && i < A.sums_met) tcg::mbar_expect_tx(bar(&sums_bar[i]), cols * nw * 16);
        if (lane < cols) {
          uint32_t to, at;
          asm("mapa.shared::cluster.u32 %0, %1, %2;"
              : "=r"(to)
              : "r"((uint32_t)__cvta_generic_to_shared(&red[i][rank][warp])), "r"(lane));
          asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(bar(&sums_bar[i])), "r"(lane));
          asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(
                           to),
                       "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(at)
                       : "memory");
        }
      } else if (lane == 0) {
        red[i][0][warp] = v;
        if (i < A.sums_met) tcg::mbar_arrive(bar(&sums_bar[i]));
      }
      __syncwarp();
    };
    auto count = [&](int i, unsigned rows) {  // of this warp, sent to barrier i
      if (lane == 0) atomicAdd(&sent[i], rows);
      if (tid == 0 && i < A.sums_met) told[i] += rows;
    };
    // A place is written again SENDS rows later: a warp that sends row x + 4 has received
    // row x + 2, so every warp has sent that, and had received row x before.  (Of a row that
    // is done again, the two exchanges alternate and are waited for at once.)
    auto send_run = [&](int i, Run r) {
      r.s += r.p.x + r.p.y;
      join_warp(r.n, r.s);
      if (TWO) {
        r.s1 += r.p1.x + r.p1.y;
        join_warp(r.n1, r.s1);
      }
      send(i, make_float4(r.n, r.s, r.n1, r.s1));
    };
    auto receive = [&](int i, uint32_t parity) {  // the same in every data thread
      wait(&sums_bar[i], parity);
      Run r;
      for (int j = lane; j < cols * MAX_WARPS; j += 32)
        if ((j & (MAX_WARPS - 1)) < nw) {
          const float4 o = red[i][j / MAX_WARPS][j & (MAX_WARPS - 1)];
          join(r.n, r.s, o.x, o.y);
          if (TWO) join(r.n1, r.s1, o.z, o.w);
        }
      join_warp(r.n, r.s);
      if (TWO) join_warp(r.n1, r.s1);
      return r;
    };

    // The first pass, a batch of the thread's pieces at a time
    auto take = [&](Run& r, const uint4* q) {
      add_pieces<T>(r.n, r.p, q, ct);
      if (TWO) add_pieces<T>(r.n1, r.p1, q, LOG2E);
    };
    uint32_t k0 = 0, k1 = 0, k2 = 0;  // slots of the copies, of the first and of the second pass
    // its row: number, place, weight, the thread's pieces, those taken, the edge and the sums
    unsigned feed_k = 0, feed_t = first;
    float feed_w = weight(first), feed_wn = weight(first + step), feed_edge = 0.f;
    int feed_n = 0, feed_whole = 0, feed_p = 0, edges = 0;
    Run feed;
    auto feed_row = [&] {  // starts on row feed_t
      const Span<T> S = span(feed_t);
      feed = Run();
      feed_p = 0;
      feed_n = feed_w != 0.f ? pieces_of(S) : 0;
      feed_whole = feed_w != 0.f ? whole_of(S) : 0;
      edges = feed_w != 0.f ? S.edges : 0;
      if (tid < edges) feed_edge = to_f32(S.row[S.edge(tid)]);
    };
    auto feed_end = [&] {  // sends row feed_t's sums, once its entries are read
      if (tid < edges) {
        add_value(feed.n, feed.p, feed_edge, ct);
        if (TWO) add_value(feed.n1, feed.p1, feed_edge, LOG2E);
      }
      if (feed_t < T0) {
        wait(&ready_bar[feed_k % BUFS], feed_k / BUFS & 1);
        if (feed_w != 0.f) send_run(feed_sent++ % SENDS, feed);
      }
      ++feed_k;
      feed_t += step;
      feed_w = feed_wn;
      feed_wn = weight(feed_t + step);
      feed_row();
    };
    auto feed_batch = [&] {
      asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD / U) : "memory");
      if (feed_p < feed_n) {
        uint4 q[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          q[u] = feed_p + u < feed_n ? from_slot(slot + k1 + u * apart) : no_piece<T>();
        take(feed, q);
      }
      advance(k1);
      feed_p += U;
      if (feed_p == A.rounds) feed_end();
    };
    // asks for and takes a row's batches where there is no second pass
    auto feed_only = [&] {
      for (int p = 0; p < A.rounds;) {
        ask_row();
        const int run = min(feed_whole - feed_p, min(ask_whole, ask_rounds)) / U;
        for (int i = 0; i < run; ++i) {
          uint4 x[U];
#pragma unroll
          for (int u = 0; u < U; ++u) copy(slot + k0 + u * apart, (const char*)ask_at + u * apart);
          asm volatile("cp.async.commit_group;" ::: "memory");
          advance(k0);
          asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD / U) : "memory");
#pragma unroll
          for (int u = 0; u < U; ++u) x[u] = from_slot(slot + k1 + u * apart);
          take(feed, x);
          advance(k1);
          ask_at += (long)U * D * N;
        }
        if (run > 0) {
          p += run * U;
          feed_p += run * U;
          ask_left -= run * U;
          ask_whole -= run * U;
          ask_rounds -= run * U;
          if (feed_p == A.rounds) feed_end();
        } else {
          ask(k0);
          advance(k0);
          feed_batch();
          p += U;
        }
      }
    };
    auto feed_direct = [&] {  // a whole row that is not held
      const Span<T> S = span(feed_t);
      for (int p = 0; p < feed_n; p += U) {
        uint4 q[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          q[u] = p + u < feed_n ? *(const uint4*)S.piece((p + u) * D + tid) : no_piece<T>();
        take(feed, q);
      }
      feed_end();
    };

    feed_row();
    if constexpr (HELD) {
      for (int p = 0; p < AHEAD; p += U) {
        ask(k0);
        advance(k0);
      }
      feed_only();
      if (GRAD)
        for (int p = 0; p < A.lead; p += U) {
          ask(k0);
          advance(k0);
          feed_batch();
        }
    } else {
      feed_direct();
    }
    float w = weight(first), wn = weight(first + step);
    int got = 0, again = 0;  // exchanges received
    unsigned k = 0;          // the CTA's rows
    for (unsigned t = first; t < T0; t += step, ++k) {
      const Span<T> S = span(t);
      const float wn2 = weight(t + 2 * step);
      const int b = k % BUFS;
      if (HELD && !GRAD) feed_only();  // without gradient the next row's first pass hides the exchange
      bool dead = w == 0.f;  // nothing to learn
      Result r = {0.f, 0.f, 0.f, 0.f, 0.f, false};
      if (!dead) {
        Run run = receive(got % SENDS, (uint32_t)(got / SENDS) & 1);
        ++got;
        // Every logit is -inf, or the largest is out of the references' reach: the sum against
        // a reference that is off by its own rounding is nothing or infinite (NaN, once joined
        // to another's); or there is a NaN.
        auto off = [](float s) { return !(s > 0.f && s < INFINITY); };
        if ((off(run.s) || (TWO && off(run.s1))) && !__any_sync(0xffffffffu, lost)) {
          const bool nan = run.s != run.s || run.s1 != run.s1;
          r.again = true;
          float top = -INFINITY;
          for (int i = tid; i < S.pieces; i += D) top = fmaxf(top, piece_max<T>(*(const uint4*)S.piece(i)));
          if (tid < S.edges) top = fmaxf(top, to_f32(S.row[S.edge(tid)]));
          const uint32_t parity = again & 1;
          ++again;
          send(SENDS, make_float4(warp_max(top), 0.f, 0.f, 0.f));
          if (CL) count(SENDS, 1);
          wait(&sums_bar[SENDS], parity);
          top = -INFINITY;
          for (int j = lane; j < cols * MAX_WARPS; j += 32)
            if ((j & (MAX_WARPS - 1)) < nw) top = fmaxf(top, red[SENDS][j / MAX_WARPS][j & (MAX_WARPS - 1)].x);
          r.top = top = warp_max(top);
          dead = top == -INFINITY && !nan;
          run = Run();
          run.n = run.n1 = 0.f;
          if (!dead) {
            auto add = [&](float v) {
              run.s += ex2((v - top) * ct);
              if (TWO) run.s1 += ex2((v - top) * LOG2E);
            };
            for (int i = tid; i < S.pieces * N; i += D) add(to_f32(S.row[S.head + i]));
            if (tid < S.edges) add(to_f32(S.row[S.edge(tid)]));
          }
          if (!__any_sync(0xffffffffu, lost)) {
            send_run(SENDS + 1, run);
            if (CL) count(SENDS + 1, 1);
          }
          run = receive(SENDS + 1, parity);
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
      if constexpr (GRAD) {
        T* dz = (T*)A.dlogits + (long)t * A.ldd + v0;
        const bool same = (((uintptr_t)dz ^ (uintptr_t)S.row) & 15) == 0;
        Factors f = {};
        if (!dead) f = factors(A, r, w, msum[b], eid[b * E1 + A.K], TWO);
        // the elements outside the pieces
        if (tid < S.edges) {
          const int e = S.edge(tid);
          dz[e] = from_f32<T>(dead ? 0.f : f.value(r, to_f32(S.row[e]), ct, TWO));
        }
        if (lane == 0) {
          own[warp].r = r;
          own[warp].f = f;
        }
        __syncwarp();
        const Gradient<T, TWO> gradient(A, r, f);
        const bool slow = gradient.slow(r, f);
        // a piece of a row that is dead or slow, or whose gradient starts elsewhere within
        // 16 bytes
        auto odd_piece = [&](uint4 x, T* out) {
          if (dead) {
            x = make_uint4(0u, 0u, 0u, 0u);
          } else {
            if (slow) {
              float2 v[N2];
              unpack<T>(x, v);
#pragma unroll
              for (int j = 0; j < N2; ++j)
                v[j] = make_float2(own[warp].f.value(own[warp].r, v[j].x, ct, TWO), own[warp].f.value(own[warp].r, v[j].y, ct, TWO));
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
        char* const out = (char*)(dz + S.head) + tid * 16;
        const int n = pieces_of(S);
        const bool plain = same && !slow;
        if constexpr (HELD) {
          const int whole = plain ? whole_of(S) : 0;
          int p = 0;
          while (p < A.rounds) {
            // batches in which every thread of the warp has its pieces of this row, of the first
            // pass's and of the one that is asked for
            ask_row();
            const int run = min(min(whole - p, feed_whole - feed_p), min(ask_whole, ask_rounds)) / U;
            if (run > 0) {
              char* o = out + (size_t)p * apart;
              const char* a = (const char*)ask_at;
              for (int i = 0; i < run; ++i) {
                uint4 x[U];
                if (!dead) {
#pragma unroll
                  for (int u = 0; u < U; ++u) x[u] = from_slot(slot + k2 + u * apart);
#pragma unroll
                  for (int u = 0; u < U; ++u) x[u] = gradient(x[u]);
                } else {
#pragma unroll
                  for (int u = 0; u < U; ++u) x[u] = make_uint4(0u, 0u, 0u, 0u);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) *(uint4*)(o + u * apart) = x[u];
#pragma unroll
                for (int u = 0; u < U; ++u) copy(slot + k2 + u * apart, a + u * apart);  // the places are free
                asm volatile("cp.async.commit_group;" ::: "memory");
                advance(k2);
                asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD / U) : "memory");
#pragma unroll
                for (int u = 0; u < U; ++u) x[u] = from_slot(slot + k1 + u * apart);
                take(feed, x);
                advance(k1);
                o += batch;
                a += batch;
              }
              p += run * U;
              feed_p += run * U;
              ask_at = (const T*)a;
              ask_left -= run * U;
              ask_whole -= run * U;
              ask_rounds -= run * U;
              if (feed_p == A.rounds) feed_end();
            } else {
              if (plain && !dead) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                  if (p + u < n) *(uint4*)(out + (size_t)(p + u) * apart) = gradient(from_slot(slot + k2 + u * apart));
              } else {
                for (int u = 0; u < U && p + u < n; ++u)
                  odd_piece(from_slot(slot + k2 + u * apart), (T*)(out + (size_t)(p + u) * apart));
              }
              ask(k2);
              advance(k2);
              feed_batch();
              p += U;
            }
          }
        } else {
          for (int p = 0; p < n; ++p) {
            const uint4 x = dead ? no_piece<T>() : *(const uint4*)S.piece(p * D + tid);
            T* o = (T*)(out + (size_t)p * apart);
            if (plain && !dead) *(uint4*)o = gradient(x);
            else odd_piece(x, o);
          }
        }
      }
      if constexpr (!HELD) feed_direct();
      __syncwarp();
      if (lane == 0 && (warp > 0 || k < A.written_met)) tcg::mbar_arrive(bar(&released_bar[b]));
      w = wn;
      wn = wn2;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (CL)
#pragma unroll 1
      for (int i = 0; i < SENDS; ++i) count(i, (feed_sent + SENDS - 1 - i) / SENDS);
  }
  // A CTA's shared memory outlives what its neighbours send: rows that were waited for have
  // landed, after a wait that gave up the rest is waited for now.
  if constexpr (CL) cooperative_groups::this_cluster().sync();
  else if constexpr (GRAD) __syncthreads();
  if constexpr (CL || GRAD) {
    bool any = false;  // the same in all of the row's CTAs
#pragma unroll
    for (int i = 0; i < MAX_TEACHERS; ++i) any |= lost_from[i] != ~0u;
    if (any) {
      if (CL && tid < SENDS + 2)
        await_sent(bar(&sums_bar[tid]), &sent[tid], told[tid], cols * nw, cols, A.wait_cycles);
      if constexpr (GRAD) {
        const int v0 = rank * A.slice;
        rows_lost<T>(lost_from, A.teachers, first, step, T0, A.weight, rank == 0 ? A.loss : nullptr, (T*)A.dlogits + v0,
                     A.ldd, min(A.slice, A.V - v0));
      }
      if constexpr (CL) cooperative_groups::this_cluster().sync();  // the others have read sent
    }
  }
}

// Rows of up to SHORT_P pieces for each thread of W warps: the row stays in registers, its
// maximum is known before its sums, and the warps of a row do everything themselves. A CTA takes one row (four rows of a warp each for the shortest) and many CTAs
// share an SM, so that their chains of loads and sums hide one another; the next CTA starts
// where one ends, since with a grid that just filled the SMs a late CTA ran alone (7929 rows
// of 1000 bf16 with 5 entries: 34 us so, 16 us now). Bound by a row's chains (its warps wait
// for one another's maxima and sums) and its instructions, 24 a column and lane in both
// directions (a fifth fewer changed 80 us to 78). At 64 registers 32 warps fit an SM (72 in
// the four-row form, which spills at 64): 5072 rows of 16384 took 78 us (74 now), and 92 us
// at 80 registers. Four pieces a thread and twice the warps: 122 us.
constexpr int SHORT_P = 8;
__host__ __device__ constexpr int short_threads(int w) { return w == 1 ? 128 : 32 * w; }

template <typename T, bool TWO, int W>
__global__ void __launch_bounds__(short_threads(W), W == 1 ? 7 : 1024 / short_threads(W))
k_distill_short(const __grid_constant__ DistillArgs A) {
  constexpr int N = Span<T>::N, N2 = N / 2, TH = 32 * W, GROUPS = short_threads(W) / TH;
  __shared__ float part[W == 1 ? 1 : 3][3][W == 1 ? 1 : W];
  const int g = threadIdx.x / TH, tid = threadIdx.x % TH, lane = tid & 31, warp = tid >> 5, E1 = A.K + 1;
  int* const id = (int*)distill_smem + g * (3 * E1 + A.table);
  float* const zj = (float*)(id + E1);
  float* const q = zj + E1;
  int* const table = (int*)(q + E1);
  auto sync = [] {
    if constexpr (W == 1) __syncwarp();
    else __syncthreads();
  };
  // three values over the row's threads, the same in each; `turn`: a place of its own
  auto over_row = [&](float (&v)[3], int turn, bool max) {
#pragma unroll
    for (int i = 0; i < 3; ++i) v[i] = max ? warp_max(v[i]) : warp_sum(v[i]);
    if constexpr (W > 1) {
      if (lane == 0)
#pragma unroll
        for (int i = 0; i < 3; ++i) part[turn][i][warp] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        v[i] = part[turn][i][0];
#pragma unroll
        for (int j = 1; j < W; ++j) v[i] = max ? fmaxf(v[i], part[turn][i][j]) : v[i] + part[turn][i][j];
      }
    } else {
      __syncwarp();
    }
  };
  const unsigned t = blockIdx.x * GROUPS + g;
  if (t < (unsigned)A.T) {
    const Span<T> S((const T*)A.logits + (long)t * A.ld, A.V);
    const float w = A.weight ? A.weight[t] : 1.f;
    const int n = (S.pieces - tid + TH - 1) / TH;
    T* dz = A.dlogits ? (T*)A.dlogits + (long)t * A.ldd : nullptr;
    const bool same = (((uintptr_t)dz ^ (uintptr_t)S.row) & 15) == 0;
    uint4 x[SHORT_P];
    float edge = -INFINITY, m[3] = {-INFINITY, -INFINITY, 0.f};  // maxima: of the row, of the entries
    bool twice = false;
    if (w != 0.f) {
#pragma unroll
      for (int p = 0; p < SHORT_P; ++p) x[p] = p < n ? *(const uint4*)S.piece(p * TH + tid) : no_piece<T>();
      if (tid < S.edges) edge = to_f32(S.row[S.edge(tid)]);
      for (int i = tid; i < A.table; i += TH) table[i] = -1;
      for (int j = tid; j <= A.K; j += TH) {
        const int e = j < A.K ? A.ids[(long)t * A.K + j] : A.labels ? A.labels[t] : -1;
        const float v = j < A.K ? A.top[(long)t * A.K + j] : 0.f;
        const bool in = e >= 0 && e < A.V, ok = in && v != -INFINITY;  // (a store's padding may hold any id)
        id[j] = ok ? e : -1;
        zj[j] = in ? to_f32(S.row[e]) : 0.f;
        q[j] = ok ? v : -INFINITY;
        if (j < A.K) m[1] = fmaxf(m[1], q[j]);
      }
      m[0] = edge;
#pragma unroll
      for (int p = 0; p < SHORT_P; ++p) m[0] = fmaxf(m[0], piece_max<T>(x[p]));
    }
    over_row(m, 0, true);
    bool dead = w == 0.f || m[0] == -INFINITY;
    // (a NaN is no maximum: a row of nothing else has the lowest one, and shows in its sums)
    const float top = m[0], tm = m[1];
    // the references are whole numbers of powers of two while they and what they are off by
    // are small enough, else the maximum is subtracted first
    const float ref = rintf(top * A.ct), ref1 = rintf(top * LOG2E);
    Result r = {ref, 0.f, TWO ? ref1 : ref, 0.f, top, !(fmaxf(fabsf(ref), TWO ? fabsf(ref1) : 0.f) <= -LOWEST)};
    float s[3] = {0.f, 0.f, 0.f};  // sums of the row at both temperatures, and of the entries
    if (w != 0.f && m[0] == -INFINITY) {
      // all -inf, or nothing but -inf and NaN
      float bad = edge != edge ? 1.f : 0.f;
#pragma unroll
      for (int p = 0; p < SHORT_P; ++p) {
        float2 v[N2];
        unpack<T>(x[p], v);
#pragma unroll
        for (int j = 0; j < N2; ++j) bad += v[j].x != v[j].x || v[j].y != v[j].y ? 1.f : 0.f;
      }
      s[0] = bad;
    }
    if (!dead) {
      float2 sum = make_float2(0.f, 0.f), sum1 = sum;
      auto add = [&](auto again) {
#pragma unroll
        for (int p = 0; p < SHORT_P; ++p)
          if (p < n) {
            float2 v[N2];
            unpack<T>(x[p], v);
#pragma unroll
            for (int j = 0; j < N2; ++j) {
              const float2 d = again ? make_float2(v[j].x - top, v[j].y - top) : v[j];
              const float2 e = again ? muls(d, both(A.ct)) : fmas(d, both(A.ct), both(-r.n));
              sum = adds(sum, make_float2(ex2(e.x), ex2(e.y)));
              if (TWO) {
                const float2 e1 = again ? muls(d, both(LOG2E)) : fmas(d, both(LOG2E), both(-r.n1));
                sum1 = adds(sum1, make_float2(ex2(e1.x), ex2(e1.y)));
              }
            }
          }
      };
      if (r.again) add(std::true_type{});
      else add(std::false_type{});
      if (tid < S.edges) {
        sum.x += ex2(r.rel(edge, A.ct));
        if (TWO) sum1.x += ex2(r.rel1(edge));
      }
      s[0] = sum.x + sum.y;
      s[1] = sum1.x + sum1.y;
      for (int j = tid; j < A.K; j += TH)
        if (id[j] >= 0) s[2] += expf((q[j] - tm) / A.tau);
    }
    over_row(s, 1, false);
    const bool nan_row = w != 0.f && m[0] == -INFINITY && s[0] > 0.f;
    r.s = nan_row ? NAN : s[0];
    r.s1 = nan_row ? NAN : TWO ? s[1] : s[0];
    if (nan_row) dead = false;
    // the entries' probabilities: a thread keeps its own
    float k[3] = {0.f, 0.f, 0.f};  // m, the divergence, entries that are repeated
    if (!dead) {
      const float lz = A.top_lse ? A.top_lse[t] - tm / A.tau : logf(s[2]), ls = logf(r.s);
      for (int j = tid; j < A.K; j += TH) {
        const float l = id[j] >= 0 ? (q[j] - tm) / A.tau - lz : -INFINITY;
        const float p = expf(l);
        q[j] = p;
        k[0] += p;
        if (p != 0.f) k[1] += p * (l - (r.rel(zj[j], A.ct) * LN2 - ls));
        if (dz && id[j] >= 0 && put_id(table, A.table, id[j])) k[2] = 1.f;
      }
    }
    over_row(k, 2, false);
    const int label = dead ? -1 : id[A.K];
    if (tid == 0) {
      float loss = 0.f;
      if (!dead) {
        loss = k[1] * A.a * A.tau * A.tau;
        if (A.b != 0.f && label >= 0) loss += A.b * (logf(r.s1) - (TWO ? r.rel1(zj[A.K]) : r.rel(zj[A.K], A.ct)) * LN2);
        loss *= w;
      }
      A.loss[t] = loss;
    }
    if (dz) {
      Factors f = {};
      if (!dead) f = factors(A, r, w, k[0], label, TWO);
      auto value = [&](float z) { return dead ? 0.f : f.value(r, z, A.ct, TWO); };
      const Gradient<T, TWO> gradient(A, r, f);
      const bool slow = gradient.slow(r, f);
#pragma unroll
      for (int p = 0; p < SHORT_P; ++p)
        if (p < n) {
          uint4 o = make_uint4(0u, 0u, 0u, 0u);
          if (slow) {
            float2 v[N2];
            unpack<T>(x[p], v);
#pragma unroll
            for (int j = 0; j < N2; ++j) v[j] = make_float2(value(v[j].x), value(v[j].y));
            o = pack<T>(v);
          } else if (!dead) {
            o = gradient(x[p]);
          }
          T* out = dz + S.head + (long)(p * TH + tid) * N;
          if (same) {
            *(uint4*)out = o;
          } else {
            const T* e = (const T*)&o;
#pragma unroll
            for (int j = 0; j < N; ++j) out[j] = e[j];
          }
        }
      if (tid < S.edges) dz[S.edge(tid)] = from_f32<T>(value(edge));
      sync();  // the dense values lie below the entries'
      twice = k[2] != 0.f;
      if (!dead)
        for (int j = tid; j <= A.K; j += TH) {
          const int e = id[j];
          if (e < 0) continue;
          const float y = entries_of(id, q, A.K, j, twice, table, A.table);
          if (y == -1.f) continue;
          dz[e] = from_f32<T>(value(zj[j]) - f.qa * y - (e == label ? f.hb : 0.f));
        }
    }
  }
}

template <typename T, bool TWO, int W>
lx_status launch_short(const DistillArgs& A, cudaStream_t s) {
  constexpr int TH = short_threads(W), GROUPS = TH / (32 * W);
  const size_t smem = (size_t)GROUPS * (3 * (A.K + 1) + A.table) * 4;
  k_distill_short<T, TWO, W><<<(A.T + GROUPS - 1) / GROUPS, TH, smem, s>>>(A);
  LX_CUDA(cudaGetLastError());
  return LX_OK;
}
template <typename T>
lx_status launch_short_any(const DistillArgs& A, cudaStream_t s) {
  const long pieces = (long)A.V * sizeof(T) / 16;
  const bool two = A.b != 0.f && A.tau != 1.f;
  // Entries a thread: with few rows one, for the row's time (64 rows of 1006 bf16, 256
  // entries: 8.2 us, 12.8 with four; 1200 rows: 18.3 and 20.4); with many four, since each
  // further warp repeats what is done once a row (7929 rows: 101 us with one, 56 with four;
  // 5072 rows of 4096, 200 entries: 65 and 43).  A single warp takes eight where the row
  // leaves it time (7929 rows of 256, 200 entries: 23 us, 39 in two warps), and one where it
  // does not (5072 rows of 2048, 100 entries: 35 us, 25 in two warps).
  const int each = A.T <= 8 * SMS ? 1 : 4;
  const int alone = each == 1 || pieces > SHORT_P * 32 / 2 ? 1 : 8;
#define LX_SHORT_CASE(W)                                                      \
  if (pieces <= SHORT_P * 32 * W && A.K <= (W == 1 ? alone : each) * 32 * W) \
    return two ? launch_short<T, true, W>(A, s) : launch_short<T, false, W>(A, s);
  LX_SHORT_CASE(1)
  LX_SHORT_CASE(2)
  LX_SHORT_CASE(4)
#undef LX_SHORT_CASE
  return two ? launch_short<T, true, 8>(A, s) : launch_short<T, false, 8>(A, s);
}

template <typename T, bool TWO, bool CL, bool HELD, bool GRAD>
lx_status launch_distill(const DistillArgs& A, int threads, int cols, int groups, size_t smem, cudaStream_t s) {
  static bool cap[64] = {};
  int dev = 0;
  LX_CUDA(cudaGetDevice(&dev));
  LX_CUDA(smem_cap_once((const void*)k_distill<T, TWO, CL, HELD, GRAD>, SMEM, dev, cap));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cols, groups);
  cfg.blockDim = dim3(threads + 32 * A.teachers);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cols;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CL ? 1 : 0;
  if (CL && cols > 2) {  // clusters that the GPCs have room for at a time: a second round would run alone
    int most = 0;
    LX_CUDA(cudaOccupancyMaxActiveClusters(&most, k_distill<T, TWO, CL, HELD, GRAD>, &cfg));
    cfg.gridDim.y = std::max(1, std::min(groups, most));
  }
  LX_CUDA(cudaLaunchKernelEx(&cfg, k_distill<T, TWO, CL, HELD, GRAD>, A));
  return LX_OK;
}

struct Shape {
  int threads, cols, groups;  // data threads of a CTA, CTAs of a row, rows at a time
  size_t smem;
};

template <typename T, bool CL, bool HELD, bool GRAD>
lx_status launch_two(const DistillArgs& A, const Shape& S, cudaStream_t s) {
  return A.b != 0.f && A.tau != 1.f ? launch_distill<T, true, CL, HELD, GRAD>(A, S.threads, S.cols, S.groups, S.smem, s)
                                    : launch_distill<T, false, CL, HELD, GRAD>(A, S.threads, S.cols, S.groups, S.smem, s);
}
template <typename T>
lx_status launch_type(const DistillArgs& A, const Shape& S, cudaStream_t s) {
  if (!A.dlogits) return S.cols > 1 ? launch_two<T, true, true, false>(A, S, s) : launch_two<T, false, true, false>(A, S, s);
  if (A.slots == 0) return launch_two<T, false, false, true>(A, S, s);
  return S.cols > 1 ? launch_two<T, true, true, true>(A, S, s) : launch_two<T, false, true, true>(A, S, s);
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
  A.sums_met = waits.unmet == LX_WAIT_CALL_SUMS ? 0 : waits.unmet == LX_WAIT_CALL_AGAIN ? SENDS : SENDS + 2;
  A.entries_met = waits.unmet == LX_WAIT_CALL_ENTRIES ? 2 : ~0u;
  A.written_met = waits.unmet == LX_WAIT_CALL_WRITTEN ? 2 : ~0u;
  A.table = 32;
  while (A.table < 2 * K) A.table *= 2;
  cudaStream_t s = (cudaStream_t)stream;
  // Rows that eight warps hold in registers.  Against the kernel with teachers' warps, us of
  // bf16 rows with gradient: 7929 x 1000, K 5: 16 and 51; 512 x 16000, K 56: 13 and 17; 5072 x
  // 16384, K 56: 74 and 87, K 300: 95 and 283, K 1000: 160 and 562; 64 x 1006, K 5: 6 either
  // way; 64 x 16384, K 512: 11 and 26.  With sixteen warps 5072 x 24000 takes 146, and 114 there.  (That
  // kernel alone has the waits.)
  if ((long)V * es / 16 <= SHORT_P * 32 * 8 && waits.unmet == LX_WAIT_NONE)
    return dtype == LX_BF16 ? launch_short_any<__nv_bfloat16>(A, s) : launch_short_any<float>(A, s);
  // CTAs of 256 data threads with half of an SM's shared memory (128 and a quarter for short
  // rows) where a row fits it, else CTAs of 512 with all of it, as many as hold a row; rows
  // too long for eight of those are not held.  Few rows are spread over more CTAs, in slices
  // of 4096 columns at least.  The shape does not depend on whether a gradient is asked for,
  // so the losses do not either.
  const bool grad = dlogits != nullptr;
  const size_t entries = ((4 * BUFS * (size_t)(K + 1) + MAX_TEACHERS * A.table + 3) / 4) * 16;
  const long row = (long)V * es;
  auto places = [&](int threads) { return ((long)SMEM * threads / 512 - (long)entries) / (16 * threads); };
  auto holds = [&](int threads) {  // bytes of a row
    return std::max(0L, (places(threads) - ahead_of(true) - U) / U * U * 16 * threads);
  };
  const bool held = row <= std::max(holds(512) * MAX_CLUSTER, holds(256));
  Shape S = {};
  S.cols = 1;
  if (held) {
    while (row > holds(256) && row > holds(512) * S.cols) S.cols *= 2;
    while (S.cols < MAX_CLUSTER && (long)T * S.cols * 2 <= SMS && V / (S.cols * 2) >= 4096) S.cols *= 2;
  }
  A.slice = S.cols == 1 ? V : ((V + S.cols - 1) / S.cols + 63) / 64 * 64;
  const long bytes = (long)A.slice * es;
  S.threads = !held || bytes > holds(256) ? 512 : bytes > holds(128) ? 256 : 128;
  A.teachers = S.threads == 512 ? MAX_TEACHERS : 2;
  A.log_d = S.threads == 512 ? 9 : S.threads == 256 ? 8 : 7;
  A.rounds = std::max(U, (int)((bytes / 16 + S.threads - 1) / S.threads + U - 1) / U * U);
  const long room = (places(S.threads) - A.rounds - ahead_of(true)) / U * U;
  A.lead = (int)std::max<long>(U, std::min<long>({LEAD, A.rounds, room}));
  A.slots = !grad ? ahead_of(false) + U : held ? A.rounds + A.lead + ahead_of(true) : 0;
  S.smem = entries + (size_t)16 * S.threads * A.slots;
  const int ctas = std::max(1, std::min((int)(65536 / (REGS * (S.threads + 32 * A.teachers))), (int)(227 * 1024 / (S.smem + 14 * 1024))));
  S.groups = std::min(T, std::max(1, SMS * ctas / S.cols));
  return dtype == LX_BF16 ? launch_type<__nv_bfloat16>(A, S, s) : launch_type<float>(A, S, s);
}
