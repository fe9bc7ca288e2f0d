// The norms around a block, with its gate and residual (lx_residual_norm):
//   s1 = (mean y^2 + eps)^-1/2,  u = y s1 (o + w_post)      (w_post NULL: u = y)
//   r' = a r + g u
//   s2 = (mean r'^2 + eps)^-1/2, h = r' s2 (o + w_pre)
// and its gradients (lx_residual_norm_backward).  With x = r' s2, n = y s1,
// W1 = o + w_post, W2 = o + w_pre and e = dh W2:
//   D  = dr' + s2 (e - x mean(e x)),   dr = a D,   dg = D u summed over what g is
//   shared by,   f = g D W1,   dy = s1 (f - n mean(f n)),
//   dw_post = sum_t g D n,   dw_pre = sum_t dh x.
//
// Both are bound by memory: a row is read once, so the forward moves r, y (and a full
// gate), r' and h, the backward r, y, dr', dh, dr and dy; r' is formed again from r and
// y instead of being read, which costs no bytes and keeps the unrounded values.
//
// A row is held by a part of a warp (H <= 256), a CTA (H <= 4096) or a cluster of CTAs,
// 8 elements a thread (16 above 32768).  Rows are dealt to a resident grid; a thread
// copies its own pieces of the next rows into slots of shared memory that it alone
// reads (cp.async: no barrier), so that two rows are in flight while one is worked on,
// and keeps its columns' parameters in registers.  In the backward it also keeps their
// gradient sums there; the CTAs' sums are added in order by a second launch, so results
// do not change from run to run.
#include <algorithm>

#include "lx_rows.cuh"

namespace lx {
namespace {

using namespace rows;

constexpr int WARP_H = 256;       // widest row of a warp
constexpr int CTA_T = 512;        // threads of a CTA at most
constexpr int CTA_H = CTA_T * 8;  // widest row of a CTA with 8 elements a thread
constexpr int MAX_CLUSTER = 8;
static_assert(2 * CTA_H * MAX_CLUSTER == LX_MAX_WIDTH, "the widest row: 16 elements a thread");
constexpr int WARP_T = 256;  // threads of a CTA whose rows are held by parts of warps

// Row arrays that are read
enum In { IN_Y = 0, IN_R = 1, IN_GATE = 2, IN_DR = 3, IN_DH = 4, N_IN = 5 };

struct NormArgs {
  int T, H, gate_kind;
  int lanes;              // threads that hold a row's piece (a part of a warp; else the CTA)
  const void* in[N_IN];   // NULL where absent
  long ld[N_IN];
  int slot[N_IN];         // place among the present ones
  int slots, stages, par_at;      // stages: rows in the slots of a thread, 3 or 2
  const float* gate;      // channel or token gate
  long ldg;
  const float *w_post, *w_pre;
  float a, off, eps;
  void *r_out, *h_out;
  float* stats;  // [2][T]: s1, s2
  // backward
  void *dr, *dy, *dgate;
  int sums;     // bits of the parameter gradients: dw_post, dgate (channel), dw_pre
  float* part;  // [CTAs of a column range][3][H]: their sums
};

// Registers a thread: the launch bounds below hold the compiler to these
constexpr int FWD_REGS = 64, BWD_REGS = 96, WIDE_REGS = 128;

enum Group { WARP = 0, CTA = 1, CLUSTER = 2 };

template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
  const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
  if constexpr (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(d), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// The rows and columns of a thread, and the slots of its pieces.  Pieces are VEC
// elements: 16 bytes, 4 bytes where rows do not start on 16-byte boundaries, or single
// bf16 values, which cannot be copied asynchronously and are read where they are used
// (as are the widest rows, whose slots would not fit).
template <typename T, int VEC, int EPT, int GRP>
struct Rows {
  static constexpr int NCH = EPT / VEC, BYTES = VEC * sizeof(T);
  static constexpr bool RING = BYTES >= 4 && EPT == 8;
  const NormArgs& A;
  char* ring;
  int lane, size, col0, end;
  int count;       // pieces of the thread inside the row (they ascend)
  long row, step;  // first row; distance of this group's rows
  __device__ Rows(const NormArgs& args, char* smem) : A(args), ring(smem) {
    col0 = 0;
    if constexpr (GRP == WARP) {
      size = A.lanes;
      lane = threadIdx.x & (size - 1);
      row = (long)blockIdx.x * (WARP_T / size) + threadIdx.x / size;
      step = (long)gridDim.x * (WARP_T / size);
    } else {
      size = blockDim.x;
      lane = threadIdx.x;
      if constexpr (GRP == CLUSTER) col0 = blockIdx.x * (CTA_T * EPT);
      row = GRP == CTA ? blockIdx.x : blockIdx.y;
      step = GRP == CTA ? gridDim.x : gridDim.y;
    }
    end = GRP == CLUSTER ? min(A.H, col0 + CTA_T * EPT) : A.H;
    count = 0;
#pragma unroll
    for (int c = 0; c < NCH; ++c) count += col(c) < end;
  }
  // whether some row of this warp (for CTAs: this CTA) is left at round `t` of lane 0
  __device__ bool more(long t) const {
    if constexpr (GRP == WARP) return __any_sync(0xffffffffu, t < A.T);
    else return t < A.T;
  }
  __device__ int col(int c) const { return col0 + (c * size + lane) * VEC; }
  __device__ const T* src(int k, long t, int e) const { return (const T*)A.in[k] + t * A.ld[k] + e; }
  __device__ char* place(int stage, int k, int c) const {
    return ring + ((size_t)((stage * A.slots + A.slot[k]) * NCH + c) * blockDim.x + threadIdx.x) * BYTES;
  }
  __device__ void fetch(int stage, long t) const {
    if constexpr (RING) {
      if (t < A.T)
#pragma unroll
        for (int k = 0; k < N_IN; ++k)
          if (A.in[k]) {
            const T* p = src(k, t, col(0));
            char* d = place(stage, k, 0);
#pragma unroll
            for (int c = 0; c < NCH; ++c, p += size * VEC, d += blockDim.x * BYTES)
              if (c < count) copy_async<BYTES>(d, p);
          }
      copy_commit();
    }
  }
  // the pieces of array k of row t, zero outside the row
  __device__ void read(int stage, int k, long t, float* v) const {
    const char* p = RING ? place(stage, k, 0) : nullptr;
    const T* g = RING ? nullptr : src(k, t, col(0));
#pragma unroll
    for (int c = 0; c < NCH; ++c, p += blockDim.x * BYTES, g += size * VEC) {
      const bool on = c < count && t < A.T;
      if constexpr (RING) {
        if constexpr (BYTES == 16) {
          load<T, VEC>((const T*)p, v + c * VEC);
        } else if constexpr (VEC == 1) {
          v[c] = *(const float*)p;
        } else {
          const uint32_t w = *(const uint32_t*)p;
          v[2 * c] = __uint_as_float(w << 16);
          v[2 * c + 1] = __uint_as_float(w & 0xffff0000u);
        }
        if (!on)
#pragma unroll
          for (int j = 0; j < VEC; ++j) v[c * VEC + j] = 0.f;
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[c * VEC + j] = 0.f;
        if (on) {
          if constexpr (BYTES == 4 && VEC == 2) {
            const uint32_t w = *(const uint32_t*)g;
            v[2 * c] = __uint_as_float(w << 16);
            v[2 * c + 1] = __uint_as_float(w & 0xffff0000u);
          } else {
            load<T, VEC>(g, v + c * VEC);
          }
        }
      }
    }
  }
  // starts the copies of the first rows; then, each round: those of the row stages - 1
  // rounds ahead, and a wait for this round's
  __device__ void begin() const {
    for (int p = 0; p < A.stages - 1; ++p) fetch(p, row + p * step);
  }
  __device__ void advance(int stage, long t) const {
    if constexpr (RING) {
      fetch(stage == 0 ? A.stages - 1 : stage - 1, t + (A.stages - 1) * step);
      if (A.stages == 3) copy_wait<2>();
      else copy_wait<1>();
    }
  }
  __device__ void write(void* out, long t, const float* v) const {
    if (t >= A.T) return;
    T* p = (T*)out + t * A.H + col(0);
#pragma unroll
    for (int c = 0; c < NCH; ++c, p += size * VEC)
      if (c < count) {
        if constexpr (BYTES == 4 && VEC == 2) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * c], v[2 * c + 1]);
          *(__nv_bfloat162*)p = b;
        } else {
          store<T, VEC>(p, v + c * VEC);
        }
      }
  }
  // fp32 parameters of the thread's columns, `rest` outside
  __device__ void params(const float* p, float add, float rest, float* v) const {
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[c * VEC + j] = p && c < count ? add + p[col(c) + j] : rest;
  }
  // sums of N values over the row's threads, the same in each of them; buf (zero at
  // first) is used in turn: a half is written again only after the barrier that follows
  // its last reads
  template <int N>
  __device__ void sum(float (&v)[N], float (*buf)[N][CTA_T / 32], int& turn) const {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      if (GRP == WARP && o >= size) continue;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
    if constexpr (GRP != WARP) {
      const int nw = blockDim.x >> 5;
      float(*b)[CTA_T / 32] = buf[turn & 1];
      ++turn;
      if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) b[i][threadIdx.x >> 5] = v[i];
      if constexpr (GRP == CTA) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.f;
#pragma unroll
        for (int w = 0; w < CTA_T / 32; w += 4)
          if (w < nw)
#pragma unroll
            for (int i = 0; i < N; ++i) {
              const float4 p = *(const float4*)&b[i][w];
              v[i] += (p.x + p.y) + (p.z + p.w);
            }
      } else {
        cooperative_groups::cluster_group cl = cooperative_groups::this_cluster();
        cl.sync();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.f;
        for (unsigned c = 0; c < cl.num_blocks(); ++c) {
          const float* q = cl.map_shared_rank(&b[0][0], c);
#pragma unroll
          for (int i = 0; i < N; ++i)
            for (int w = 0; w < nw; ++w) v[i] += q[i * (CTA_T / 32) + w];
        }
      }
    }
  }
};

template <int N>
__device__ __forceinline__ void clear(float (*buf)[N][CTA_T / 32]) {
  for (int i = threadIdx.x; i < 2 * N * (CTA_T / 32); i += blockDim.x) (&buf[0][0][0])[i] = 0.f;
  __syncthreads();
}

extern __shared__ uint4 norm_ring[];

template <typename T, int VEC, int EPT, int GRP>
__global__ void __launch_bounds__(CTA_T, EPT == 8 ? 2 : 1)
k_resnorm_fwd(const NormArgs A) {
  __shared__ __align__(16) float buf[2][1][CTA_T / 32];
  int turn = 0;
  if (GRP == CTA) clear(buf);
  const Rows<T, VEC, EPT, GRP> R(A, (char*)norm_ring);
  const float inv = 1.f / (float)A.H;
  const bool chan = A.gate_kind == LX_GATE_CHANNEL;
  float w1[EPT], w2[EPT];  // w1: with the channel gate
  R.params(A.w_post, A.off, 1.f, w1);
  R.params(A.w_pre, A.off, 0.f, w2);
  if (chan) {
    float g[EPT];
    R.params(A.gate, 0.f, 0.f, g);
#pragma unroll
    for (int i = 0; i < EPT; ++i) w1[i] *= g[i];
  }
  int stage = 0;
  R.begin();
  const bool token = A.gate_kind == LX_GATE_TOKEN;
  float next = token && R.row < A.T ? A.gate[R.row * A.ldg] : 1.f;  // a row's gate is read a round ahead
  for (long t = R.row; R.more(t); t += R.step) {
    const float tok = next;
    if (token && t + R.step < A.T) next = A.gate[(t + R.step) * A.ldg];
    R.advance(stage, t);
    float x[EPT];
    R.read(stage, IN_R, t, x);
    float s1 = 1.f, s2 = 1.f, q[1];
    if (A.in[IN_Y]) {
      float y[EPT];
      R.read(stage, IN_Y, t, y);
      if (A.w_post) {
        q[0] = 0.f;
#pragma unroll
        for (int i = 0; i < EPT; ++i) q[0] = fmaf(y[i], y[i], q[0]);
        R.sum(q, buf, turn);
        s1 = rsqrtf(q[0] * inv + A.eps);
      }
      if (A.in[IN_GATE]) {
        float g[EPT];
        R.read(stage, IN_GATE, t, g);
#pragma unroll
        for (int i = 0; i < EPT; ++i) y[i] *= g[i];
      }
      const float f = s1 * tok;
#pragma unroll
      for (int i = 0; i < EPT; ++i) x[i] = fmaf(y[i] * w1[i], f, A.a * x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < EPT; ++i) x[i] *= A.a;
    }
    if (A.r_out) R.write(A.r_out, t, x);
    if (A.w_pre) {
      q[0] = 0.f;
#pragma unroll
      for (int i = 0; i < EPT; ++i) q[0] = fmaf(x[i], x[i], q[0]);
      R.sum(q, buf, turn);
      s2 = rsqrtf(q[0] * inv + A.eps);
#pragma unroll
      for (int i = 0; i < EPT; ++i) x[i] *= s2 * w2[i];
      R.write(A.h_out, t, x);
    }
    if (A.stats && R.lane == 0 && R.col0 == 0 && t < A.T) {
      A.stats[t] = s1;
      A.stats[(long)A.T + t] = s2;
    }
    stage = stage + 1 == A.stages ? 0 : stage + 1;
  }
  // a CTA's shared memory outlives its neighbours' reads
  if constexpr (GRP == CLUSTER) cooperative_groups::this_cluster().sync();
}

// With x, D0 = dr' + s2 e and v = g u in hand, one set of sums serves both norms:
// mean(e x) gives D = D0 - m x, and sum(f n) = sum(D v) = sum(D0 v) - m sum(x v) (for a
// token's gate the sums are of u, which its gradient needs, and f n is g times them).
template <typename T, int VEC, int EPT, int GRP>
__global__ void __launch_bounds__(EPT == 8 ? 640 : CTA_T, 1)
k_resnorm_bwd(const NormArgs A) {
  __shared__ __align__(16) float buf[2][3][CTA_T / 32];
  int turn = 0;
  if (GRP == CTA) clear(buf);
  const Rows<T, VEC, EPT, GRP> R(A, (char*)norm_ring);
  const float inv = 1.f / (float)A.H;
  const bool token = A.gate_kind == LX_GATE_TOKEN;
  // the columns' parameters, in slots that only this thread reads: registers are short
  float4* par = (float4*)((char*)norm_ring + A.par_at);
  auto put = [&](int k, const float* v) {
#pragma unroll
    for (int i = 0; i < EPT; i += 4)
      par[(k * (EPT / 4) + i / 4) * blockDim.x + threadIdx.x] = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  };
  auto get = [&](int k, float* v) {
#pragma unroll
    for (int i = 0; i < EPT; i += 4) {
      const float4 p = par[(k * (EPT / 4) + i / 4) * blockDim.x + threadIdx.x];
      v[i] = p.x;
      v[i + 1] = p.y;
      v[i + 2] = p.z;
      v[i + 3] = p.w;
    }
  };
  {
    float v[EPT];
    R.params(A.w_post, A.off, 1.f, v);
    put(0, v);
    R.params(A.w_pre, A.off, 0.f, v);
    put(1, v);
    R.params(A.gate_kind == LX_GATE_CHANNEL ? A.gate : nullptr, 0.f, 1.f, v);
    put(2, v);
  }
  float acc[3][EPT];
#pragma unroll
  for (int i = 0; i < EPT; ++i) acc[0][i] = acc[1][i] = acc[2][i] = 0.f;
  int stage = 0;
  R.begin();
  float n1 = 0.f, n2 = 0.f, ng = 1.f;  // a row's scalars are read a round ahead
  auto scalars = [&](long t) {
    if (t >= A.T) return;
    n1 = A.stats[t];
    n2 = A.stats[(long)A.T + t];
    if (token) ng = A.gate[t * A.ldg];
  };
  scalars(R.row);
  for (long t = R.row; R.more(t); t += R.step) {
    const bool on = t < A.T;
    const float s1 = n1, s2 = n2, tok = ng;
    scalars(t + R.step);
    R.advance(stage, t);
    float n[EPT], D[EPT], x[EPT], g[EPT];  // n: y s1
    if (A.in[IN_DR]) R.read(stage, IN_DR, t, D);
    else
#pragma unroll
      for (int i = 0; i < EPT; ++i) D[i] = 0.f;
    if (A.in[IN_Y]) {
      R.read(stage, IN_Y, t, n);
#pragma unroll
      for (int i = 0; i < EPT; ++i) n[i] *= s1;
      if (A.in[IN_GATE]) {
        R.read(stage, IN_GATE, t, g);
      } else {
#pragma unroll
        for (int i = 0; i < EPT; ++i) g[i] = 1.f;
        if (A.gate_kind == LX_GATE_CHANNEL) get(2, g);
      }
    }
    float w1[EPT];
    get(0, w1);
    float q[3] = {0.f, 0.f, 0.f};
    if (A.in[IN_DH]) {
      float dh[EPT], w2[EPT];
      get(1, w2);
      R.read(stage, IN_R, t, x);
      R.read(stage, IN_DH, t, dh);
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        float v = A.a * x[i];
        if (A.in[IN_Y]) v = fmaf(n[i] * w1[i], g[i] * tok, v);
        x[i] = v * s2;
        acc[2][i] = fmaf(dh[i], x[i], acc[2][i]);
        const float e = dh[i] * w2[i];
        q[0] = fmaf(e, x[i], q[0]);
        D[i] = fmaf(s2, e, D[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPT; ++i) x[i] = 0.f;
    }
    if (A.in[IN_Y]) {
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        const float v = n[i] * w1[i] * g[i];
        q[1] = fmaf(D[i], v, q[1]);
        q[2] = fmaf(x[i], v, q[2]);
      }
    }
    R.sum(q, buf, turn);
    const float m = q[0] * inv * s2;
    const float dv = q[1] - m * q[2];
    const float m1 = A.w_post ? dv * inv * tok : 0.f;
#pragma unroll
    for (int i = 0; i < EPT; ++i) D[i] = fmaf(-m, x[i], D[i]);
    if (A.dr) {
#pragma unroll
      for (int i = 0; i < EPT; ++i) x[i] = A.a * D[i];
      R.write(A.dr, t, x);
    }
    if (A.in[IN_Y]) {
      if (token && A.dgate && R.lane == 0 && R.col0 == 0 && on) ((float*)A.dgate)[t] = dv;
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        x[i] = D[i] * (n[i] * w1[i]);
        acc[1][i] += x[i];
        const float f = D[i] * (g[i] * tok);
        acc[0][i] = fmaf(f, n[i], acc[0][i]);
        D[i] = s1 * fmaf(-m1, n[i], f * w1[i]);
      }
      if (A.in[IN_GATE] && A.dgate) R.write(A.dgate, t, x);
      if (A.dy) R.write(A.dy, t, D);
    }
    stage = stage + 1 == A.stages ? 0 : stage + 1;
  }
  if (A.part) {
    float* part = A.part + (GRP == CLUSTER ? (long)blockIdx.y : (long)blockIdx.x) * 3 * A.H;
    float* ws = (float*)norm_ring;  // [rows of the CTA][H], the ring's copies being done
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      if (!(A.sums >> k & 1)) continue;
      if constexpr (GRP == WARP) {
        copy_wait<0>();
        __syncthreads();
#pragma unroll
        for (int c = 0; c < R.NCH; ++c)
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            if (R.col(c) + j < A.H) ws[(threadIdx.x / R.size) * A.H + R.col(c) + j] = acc[k][c * VEC + j];
        __syncthreads();
        for (int e = threadIdx.x; e < A.H; e += WARP_T) {
          float s = 0.f;
          for (int w = 0; w < WARP_T / R.size; ++w) s += ws[w * A.H + e];
          part[(long)k * A.H + e] = s;
        }
      } else {
#pragma unroll
        for (int c = 0; c < R.NCH; ++c)
          if (R.col(c) < R.end)
#pragma unroll
            for (int j = 0; j < VEC; ++j) part[(long)k * A.H + R.col(c) + j] = acc[k][c * VEC + j];
      }
    }
  }
  if constexpr (GRP == CLUSTER) cooperative_groups::this_cluster().sync();
}

// out[k][e] = sum over p of part[p][k][e], in a fixed order: 32 columns and 8 ranges
// of p a CTA
__global__ void __launch_bounds__(256)
k_resnorm_sum(const float* __restrict__ part, int n, int H, float* o0, float* o1, float* o2) {
  __shared__ float sm[8][32];
  const int k = blockIdx.y, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  float* out = k == 0 ? o0 : k == 1 ? o1 : o2;
  if (!out) return;
  const int e = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (e < H)
#pragma unroll 8
    for (int p = w; p < n; p += 8) s += part[((long)p * 3 + k) * H + e];
  sm[w][lane] = s;
  __syncthreads();
  if (w == 0 && e < H) {
#pragma unroll
    for (int i = 1; i < 8; ++i) s += sm[i][lane];
    out[e] = s;
  }
}

struct Shape {
  int grp, ept, threads, cols, lanes;  // cols: CTAs to a row
  long groups;                         // CTAs (clusters) that have a row
};

Shape shape_of(int T, int H) {
  Shape s;
  s.grp = H <= WARP_H ? WARP : H <= CTA_H ? CTA : CLUSTER;
  s.ept = H <= CTA_H * MAX_CLUSTER ? 8 : 16;
  s.cols = s.grp == CLUSTER ? (H + CTA_T * s.ept - 1) / (CTA_T * s.ept) : 1;
  s.lanes = 1;
  while (s.lanes < 32 && s.lanes * 8 < H) s.lanes *= 2;
  s.threads = s.grp == WARP ? WARP_T : s.grp == CTA ? (H + 255) / 256 * 32 : CTA_T;
  s.groups = s.grp == WARP ? ((long)T + WARP_T / s.lanes - 1) / (WARP_T / s.lanes) : T;
  return s;
}

constexpr int SMS = 152;

// CTAs (clusters) that rows are dealt to: what is resident with `regs` registers a
// thread and `smem` bytes a CTA
long resident(const Shape& s, int regs, size_t smem) {
  const long ctas = std::min<long>(65536 / (regs * s.threads), (long)(227 * 1024 / (smem + 2048)));
  return std::min(s.groups, std::max(1L, SMS * std::max(1L, ctas) / s.cols));
}

// The backward's groups fix the workspace: they do not depend on types or strides
long bwd_groups(const Shape& s) { return resident(s, s.ept == 8 ? BWD_REGS : WIDE_REGS, 0); }

// Slots of a CTA: three rows, or two where three would keep CTAs off an SM that its
// registers have room for (fp32 with a full gate)
size_t ring_bytes(const Shape& s, NormArgs& A, size_t es, int regs, size_t more) {
  const size_t row = (size_t)A.slots * s.ept * es * s.threads;
  A.stages = (3 * row + more + 1024) * (65536 / (regs * s.threads)) <= 227 * 1024 ? 3 : 2;
  return A.stages * row;
}

template <typename... KArgs>
lx_status launch(void (*kern)(KArgs...), const Shape& s, long groups, size_t smem, const NormArgs& A, cudaStream_t st,
                 bool (&cap)[64]) {
  int dev = 0;
  LX_CUDA(cudaGetDevice(&dev));
  LX_CUDA(smem_cap_once((const void*)kern, 224 * 1024, dev, cap));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = s.grp == CLUSTER ? dim3(s.cols, (unsigned)groups) : dim3((unsigned)groups);
  cfg.blockDim = dim3(s.threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = s.cols;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = s.grp == CLUSTER ? 1 : 0;
  LX_CUDA(cudaLaunchKernelEx(&cfg, kern, A));
  return LX_OK;
}

template <typename T, int VEC, int EPT, int GRP, bool BWD>
lx_status launch_one(const Shape& s, NormArgs& A, cudaStream_t st) {
  static bool cap[64] = {};
  constexpr int REGS = EPT == 16 ? WIDE_REGS : BWD ? BWD_REGS : FWD_REGS;
  const size_t par = BWD ? sizeof(float) * 3 * EPT * s.threads : 0;
  size_t smem = 0;
  A.stages = 2;
  if (VEC * sizeof(T) >= 4 && EPT == 8) smem = ring_bytes(s, A, sizeof(T), REGS, par);
  A.par_at = (int)smem;
  smem += par;
  if (BWD && GRP == WARP) smem = std::max(smem, sizeof(float) * (WARP_T / s.lanes) * A.H);
  if (BWD) return launch(k_resnorm_bwd<T, VEC, EPT, GRP>, s, bwd_groups(s), smem, A, st, cap);
  return launch(k_resnorm_fwd<T, VEC, EPT, GRP>, s, resident(s, REGS, smem), smem, A, st, cap);
}

template <typename T, int VEC, bool BWD>
lx_status launch_vec(const Shape& s, NormArgs& A, cudaStream_t st) {
  if (s.grp == WARP) return launch_one<T, VEC, 8, WARP, BWD>(s, A, st);
  if (s.grp == CTA) return launch_one<T, VEC, 8, CTA, BWD>(s, A, st);
  if (s.ept == 8) return launch_one<T, VEC, 8, CLUSTER, BWD>(s, A, st);
  return launch_one<T, VEC, 16, CLUSTER, BWD>(s, A, st);
}

// piece: bytes that divide every row's start and length (16, 4, or 2)
template <bool BWD>
lx_status launch_any(int dtype, int piece, const Shape& s, NormArgs& A, cudaStream_t st) {
  if (dtype == LX_F32)
    return piece == 16 ? launch_vec<float, 4, BWD>(s, A, st) : launch_vec<float, 1, BWD>(s, A, st);
  if (piece == 16) return launch_vec<__nv_bfloat16, 8, BWD>(s, A, st);
  if (piece == 4) return launch_vec<__nv_bfloat16, 2, BWD>(s, A, st);
  return launch_vec<__nv_bfloat16, 1, BWD>(s, A, st);
}

size_t esize(int dtype) { return dtype == LX_BF16 ? 2 : 4; }

lx_status check_desc(const lx_resnorm_desc* d) {
  if (!d) return fail(LX_ERR_ARG, "desc is NULL");
  if (d->dtype != LX_F32 && d->dtype != LX_BF16) return fail(LX_ERR_ARG, "unknown dtype");
  if (d->T < 0) return fail(LX_ERR_ARG, "T < 0");
  if (d->H < 1 || d->H > LX_MAX_WIDTH) return fail(LX_ERR_SHAPE, "H must be in 1..LX_MAX_WIDTH");
  if (d->gate_kind < LX_GATE_NONE || d->gate_kind > LX_GATE_FULL) return fail(LX_ERR_ARG, "unknown gate kind");
  if (!(d->eps >= 0.f)) return fail(LX_ERR_ARG, "eps must not be negative");
  if (d->T == 0) return LX_OK;  // pointers to nothing
  if (!d->y && (d->w_post || d->gate_kind != LX_GATE_NONE)) return fail(LX_ERR_ARG, "w_post and a gate need y");
  if (!d->y && !d->w_pre) return fail(LX_ERR_ARG, "y and w_pre are both NULL");
  if ((d->gate_kind != LX_GATE_NONE) != (d->gate != nullptr)) return fail(LX_ERR_ARG, "gate does not match gate_kind");
  if (!d->r) return fail(LX_ERR_ARG, "r is NULL");
  if (d->ldr < d->H || (d->y && d->ldy < d->H) || (d->gate_kind == LX_GATE_FULL && d->ldg < d->H) ||
      (d->gate_kind == LX_GATE_TOKEN && d->ldg < 0))
    return fail(LX_ERR_SHAPE, "rows are closer than H elements");
  const size_t es = esize(d->dtype);
  if (!aligned(d->r, es) || !aligned(d->y, es) || !aligned(d->gate, d->gate_kind == LX_GATE_FULL ? es : 4) ||
      !aligned(d->w_post, 4) || !aligned(d->w_pre, 4))
    return fail(LX_ERR_ARG, "a pointer is not aligned to its element");
  return LX_OK;
}

NormArgs args_of(const lx_resnorm_desc* d, const Shape& s) {
  NormArgs A = {};
  A.T = d->T;
  A.H = d->H;
  A.gate_kind = d->gate_kind;
  A.lanes = s.lanes;
  A.in[IN_Y] = d->y;
  A.ld[IN_Y] = d->ldy;
  A.in[IN_R] = d->r;
  A.ld[IN_R] = d->ldr;
  if (d->gate_kind == LX_GATE_FULL) {
    A.in[IN_GATE] = d->gate;
    A.ld[IN_GATE] = d->ldg;
  } else {
    A.gate = (const float*)d->gate;
    A.ldg = d->ldg;
  }
  A.w_post = d->w_post;
  A.w_pre = d->w_pre;
  A.a = d->res_scale;
  A.off = d->weight_offset;
  A.eps = d->eps;
  return A;
}

// Numbers the arrays that are read and finds the widest piece that divides every row's
// start and length: 16 bytes, 4, or one bf16
int pieces(NormArgs& A, size_t es, std::initializer_list<const void*> outs) {
  uintptr_t bits = (uintptr_t)A.H * es;
  A.slots = 0;
  for (int k = 0; k < N_IN; ++k)
    if (A.in[k]) {
      A.slot[k] = A.slots++;
      bits |= (uintptr_t)A.in[k] | (uintptr_t)((size_t)A.ld[k] * es);
    }
  for (const void* p : outs) bits |= (uintptr_t)p;
  return bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 2;
}

}  // namespace
}  // namespace lx

extern "C" lx_status lx_residual_norm(const lx_resnorm_desc* d, void* r_out, void* h_out, float* stats,
                                      void* stream) {
  using namespace lx;
  LX_TRY(check_desc(d));
  if (d->T == 0) return LX_OK;
  if ((h_out != nullptr) != (d->w_pre != nullptr)) return fail(LX_ERR_ARG, "h_out goes with w_pre");
  if (!r_out && !h_out) return fail(LX_ERR_ARG, "r_out and h_out are both NULL");
  const size_t es = esize(d->dtype), out = (size_t)d->T * d->H * es;
  if (!aligned(r_out, es) || !aligned(h_out, es) || !aligned(stats, 4))
    return fail(LX_ERR_ARG, "a pointer is not aligned to its element");
  const size_t sr = span(d->T, d->H, d->ldr, es), sy = span(d->T, d->H, d->ldy, es);
  const size_t sg = d->gate_kind == LX_GATE_FULL    ? span(d->T, d->H, d->ldg, es)
                    : d->gate_kind == LX_GATE_TOKEN ? span(d->T, 1, d->ldg, 4)
                                                    : 4 * (size_t)d->H;
  const bool in_place = r_out == d->r && d->ldr == d->H;
  if ((!in_place && overlap(r_out, out, d->r, sr)) || overlap(r_out, out, d->y, sy) || overlap(r_out, out, d->gate, sg) ||
      overlap(h_out, out, d->r, sr) || overlap(h_out, out, d->y, sy) || overlap(h_out, out, d->gate, sg) ||
      overlap(r_out, out, h_out, out))
    return fail(LX_ERR_ARG, "an output overlaps an input");
  const Shape s = shape_of(d->T, d->H);
  NormArgs A = args_of(d, s);
  A.r_out = r_out;
  A.h_out = h_out;
  A.stats = stats;
  return launch_any<false>(d->dtype, pieces(A, es, {r_out, h_out}), s, A, (cudaStream_t)stream);
}

extern "C" lx_status lx_residual_norm_workspace(int32_t T, int32_t H, uint64_t* bytes) {
  using namespace lx;
  if (!bytes) return fail(LX_ERR_ARG, "bytes is NULL");
  if (T < 0) return fail(LX_ERR_ARG, "T < 0");
  if (H < 1 || H > LX_MAX_WIDTH) return fail(LX_ERR_SHAPE, "H must be in 1..LX_MAX_WIDTH");
  *bytes = (uint64_t)bwd_groups(shape_of(T, H)) * 3 * H * sizeof(float);
  return LX_OK;
}

extern "C" lx_status lx_residual_norm_backward(const lx_resnorm_desc* d, const float* stats, const void* dr_out,
                                               int64_t lddr, const void* dh, int64_t lddh, void* dr, void* dy,
                                               float* dw_post, void* dgate, float* dw_pre, void* workspace,
                                               uint64_t workspace_bytes, void* stream) {
  using namespace lx;
  LX_TRY(check_desc(d));
  if (dw_post && !d->w_post) return fail(LX_ERR_ARG, "dw_post goes with w_post");
  if (dw_pre && !d->w_pre) return fail(LX_ERR_ARG, "dw_pre goes with w_pre");
  if (dgate && d->gate_kind == LX_GATE_NONE) return fail(LX_ERR_ARG, "dgate goes with a gate");
  if (dy && !d->y) return fail(LX_ERR_ARG, "dy goes with y");
  if (dh && !d->w_pre) return fail(LX_ERR_ARG, "dh goes with w_pre");
  const size_t es = esize(d->dtype), out = (size_t)d->T * d->H * es;
  if (!aligned(dr_out, es) || !aligned(dh, es) || !aligned(dr, es) || !aligned(dy, es) || !aligned(dw_post, 4) ||
      !aligned(dw_pre, 4) || !aligned(stats, 4) || !aligned(dgate, d->gate_kind == LX_GATE_FULL ? es : 4))
    return fail(LX_ERR_ARG, "a pointer is not aligned to its element");
  float* dgc = d->gate_kind == LX_GATE_CHANNEL ? (float*)dgate : nullptr;
  const bool params = dw_post || dw_pre || dgc;
  cudaStream_t st = (cudaStream_t)stream;
  if (d->T == 0) {
    for (float* p : {dw_post, dw_pre, dgc})
      if (p) LX_CUDA(cudaMemsetAsync(p, 0, sizeof(float) * d->H, st));
    return LX_OK;
  }
  if (!stats) return fail(LX_ERR_ARG, "stats is NULL");
  if (!dr_out && !dh) return fail(LX_ERR_ARG, "dr_out and dh are both NULL");
  if ((dr_out && lddr < d->H) || (dh && lddh < d->H)) return fail(LX_ERR_SHAPE, "rows are closer than H elements");
  const void* ins[] = {d->r, d->y, d->gate_kind == LX_GATE_FULL ? d->gate : nullptr, dr_out, dh};
  const long lds[] = {(long)d->ldr, (long)d->ldy, (long)d->ldg, (long)lddr, (long)lddh};
  void* outs[] = {dr, dy, d->gate_kind == LX_GATE_FULL ? dgate : nullptr};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 5; ++j)
      if (overlap(outs[i], out, ins[j], span(d->T, d->H, lds[j], es)))
        return fail(LX_ERR_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], out, outs[j], out)) return fail(LX_ERR_ARG, "two outputs overlap");
  }
  const Shape s = shape_of(d->T, d->H);
  const long groups = bwd_groups(s);
  if (params) {
    if (!workspace || !aligned(workspace, 16)) return fail(LX_ERR_ARG, "workspace is NULL or not 16-byte aligned");
    if (workspace_bytes < (uint64_t)groups * 3 * d->H * sizeof(float)) return fail(LX_ERR_ARG, "workspace too small");
  }
  NormArgs A = args_of(d, s);
  if (!dh) A.in[IN_R] = nullptr;  // only the second norm's gradient reads r
  A.stats = const_cast<float*>(stats);
  A.in[IN_DR] = dr_out;
  A.ld[IN_DR] = lddr;
  A.in[IN_DH] = dh;
  A.ld[IN_DH] = lddh;
  A.dr = dr;
  A.dy = dy;
  A.dgate = dgate;
  A.part = params ? (float*)workspace : nullptr;
  A.sums = (dw_post ? 1 : 0) | (dgc ? 2 : 0) | (dw_pre ? 4 : 0);
  LX_TRY(launch_any<true>(d->dtype, pieces(A, es, {outs[0], outs[1], outs[2]}), s, A, st));
  if (params) {
    k_resnorm_sum<<<dim3((d->H + 31) / 32, 3), 256, 0, st>>>(A.part, (int)groups, d->H, dw_post, dgc, dw_pre);
    LX_CUDA(cudaGetLastError());
  }
  return LX_OK;
}
