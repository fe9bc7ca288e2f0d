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
// A row is held by a part of a warp (H <= 512), a CTA (H <= 4096) or a cluster of CTAs,
// 16 elements a thread: what a row costs besides its elements (two barriers, the sums,
// the copies' addresses) bounded the kernels with 8.  Rows are dealt to a resident grid; a thread
// copies its own pieces of the next rows into slots of shared memory that it alone
// reads (cp.async: no barrier), so that two rows are in flight while one is worked on,
// and keeps its columns' parameters in registers.  In the backward it also keeps their
// gradient sums there; the CTAs' sums are added in order by a second launch, so results
// do not change from run to run.
#include <cooperative_groups.h>

#include <algorithm>

#include "lx_rows.cuh"

namespace lx {
namespace {

using namespace rows;

constexpr int EPT = 16, N2 = EPT / 2;  // elements of a row a thread holds, in pairs
constexpr int WARP_H = 32 * EPT;       // widest row of a warp
constexpr int CTA_T = 256;             // threads of a CTA at most,
constexpr int WIDE_T = 512;            // or for the widest rows
constexpr int MAX_CLUSTER = 8;
static_assert(EPT * WIDE_T * MAX_CLUSTER == LX_MAX_WIDTH, "the widest row");

// Row arrays that are read
enum In { IN_Y = 0, IN_R = 1, IN_GATE = 2, IN_DR = 3, IN_DH = 4, N_IN = 5 };

struct NormArgs {
  int T, H, gate_kind;
  int lanes;              // threads that hold a row's piece (a part of a warp; else the CTA)
  const void* in[N_IN];   // NULL where absent
  uint32_t ldb[N_IN];     // bytes between rows
  uint32_t slot_at[N_IN]; // bytes from a stage's start to the array's slots
  uint32_t ends;          // rows at either end of the arrays whose blocks may reach beyond
  uint32_t stage_bytes, stages;  // of a CTA's slots for one row; rows they hold, 3 or 2
  uint32_t par_at;        // bytes from the slots' start to the parameters'
  const float* gate;      // channel or token gate
  long ldg;
  const float *w_post, *w_pre;
  float a, off, eps;
  void *r_out, *h_out;
  float* stats;  // [2][T]: s1, s2
  void* q_out;   // Q8: e4m3 [T][H],
  float* scale;  // and [T]
  // backward
  void *dr, *dy, *dgate;
  int sums;     // bits of the column sums wanted: of s1 D y, of dh x
  float* part;  // [CTAs of a column range][2][H]: those sums
};

constexpr int REGS = 128;  // a thread: the launch bounds hold the compiler to these

constexpr float E4M3_MAX = 448.f, TINY = 1.17549435e-38f, SMALL = 7.8886091e-31f;  // 2^-126, 2^-100

// four values in e4m3, to the nearest, what is above 448 as 448
__device__ __forceinline__ uint32_t to_e4m3(float2 a, float2 b) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(lo) : "f"(a.x), "f"(a.y));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(hi) : "f"(b.x), "f"(b.y));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}

// bytes of the slots of one array's columns of a group: `members` threads' and a block more
__host__ __device__ constexpr int group_bytes(int members, int es) { return members * EPT * es + 16; }

enum Group { WARP = 0, CTA = 1, CLUSTER = 2, WIDE = 3 };  // WIDE: a cluster of larger CTAs
constexpr int max_threads(int grp) { return grp == WIDE ? WIDE_T : CTA_T; }
constexpr int max_cols(int grp) { return grp >= CLUSTER ? MAX_CLUSTER : 1; }

__device__ __forceinline__ void copy_async(void* dst, const void* src) {
  const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
}
// the first `bytes` of 16, the rest of them zero
__device__ __forceinline__ void copy_async(void* dst, const void* src, uint32_t bytes) {
  const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// The rows and columns of a thread, and the slots of its pieces.  Where every row starts on
// a 16-byte boundary, pieces are 16 bytes (VEC elements) and a thread copies its own.
// Elsewhere (VEC = 1) a warp, or the part of one that holds a row, copies the 16-byte blocks
// that its columns of the row touch, and a thread picks every 32nd element: the shift of a
// row within its blocks is known when it is read.  (Single loads: 1031
// rows of 2047 bf16 16.5 us forward, 33.2 backward; blocks 13.6, 27.2.)  The widest rows, whose slots would not fit, are read
// where they are used.  Values are held as pairs.
template <typename T, int VEC, int GRP>
struct Rows {
  static constexpr int NCH = EPT / VEC, MAX_T = max_threads(GRP), MAX_W = MAX_T / 32;
  static constexpr bool RING = GRP != WIDE, BLOCK = RING && VEC == 1;
  static constexpr int COLS = max_cols(GRP);
  static_assert(VEC == 1 || VEC * sizeof(T) == 16, "single elements or 16 bytes");
  const NormArgs& A;
  char* ring;     // the thread's first slot (BLOCK: its group's)
  uint32_t at;    // the round's stage, in bytes
  int lane, size;  // of the threads that hold a row
  int col0;        // first column of the thread
  int count;       // its pieces inside the row (they ascend)
  int row, step;   // first row; distance of this group's rows
  __device__ Rows(const NormArgs& args, char* smem) : A(args), at(0) {
    int first = 0, end = A.H;
    if constexpr (GRP == WARP) {
      size = A.lanes;
      lane = threadIdx.x & (size - 1);
      row = blockIdx.x * (CTA_T / size) + threadIdx.x / size;
      step = gridDim.x * (CTA_T / size);
    } else {
      size = blockDim.x;
      lane = threadIdx.x;
      row = GRP == CTA ? blockIdx.x : blockIdx.y;
      step = GRP == CTA ? gridDim.x : gridDim.y;
      if constexpr (GRP >= CLUSTER) {
        first = blockIdx.x * (MAX_T * EPT);
        end = min(A.H, first + MAX_T * EPT);
      }
    }
    if constexpr (BLOCK) {
      const int group = threadIdx.x / members();
      col0 = (GRP == WARP ? 0 : first + group * 32 * EPT) + lane % members();
      ring = smem + group * group_bytes(members(), sizeof(T));
    } else {
      col0 = first + lane * VEC;
      ring = smem + threadIdx.x * 16;
    }
    count = 0;
#pragma unroll
    for (int c = 0; c < NCH; ++c) count += col(c) < end;
  }
  __device__ bool writer() const { return col0 == 0; }  // one thread of the row
  // whether a row is left for this warp (for CTAs: this CTA) in round t of lane 0; t is
  // below 2 * T, and T + step below 2^31 + 2^20: compared as unsigned
  __device__ bool more(unsigned t) const {
    if constexpr (GRP == WARP) return __any_sync(0xffffffffu, t < (unsigned)A.T);
    else return t < (unsigned)A.T;
  }
  __device__ int members() const { return GRP == WARP ? size : 32; }  // BLOCK: threads of a group
  __device__ int apart() const { return BLOCK ? members() : size * VEC; }  // columns between pieces
  __device__ int seg() const { return col0 - lane % members(); }           // BLOCK: the group's first column,
  __device__ int seg_n() const {                                           // and its columns
    const int end = GRP >= CLUSTER ? min(A.H, (int)(blockIdx.x + 1) * MAX_T * EPT) : A.H;
    return max(0, min(end - seg(), members() * EPT));
  }
  __device__ int col(int c) const { return BLOCK ? col0 + c * members() : col0 + c * size * VEC; }
  __device__ const T* src(int k, unsigned t, int col) const {
    return (const T*)((const char*)A.in[k] + (uint64_t)t * A.ldb[k]) + col;
  }
  // BLOCK: bytes from a 16-byte boundary to the group's first element
  __device__ int shift(int k, unsigned t) const {
    return ((uint32_t)(uintptr_t)A.in[k] + t * A.ldb[k] + (uint32_t)seg() * (uint32_t)sizeof(T)) & 15;
  }
  __device__ char* place(uint32_t stage, int k) const { return ring + (stage + A.slot_at[k]); }
  __device__ void fetch(uint32_t stage, unsigned t) const {
    if (t < (unsigned)A.T)
#pragma unroll
      for (int k = 0; k < N_IN; ++k)
        if (A.in[k]) {
          char* d = place(stage, k);
          if constexpr (BLOCK) {
            const int step_b = members() * 16, me = lane % members() * 16;
            const int off = shift(k, t), bytes = off + seg_n() * (int)sizeof(T);  // from the first block on
            const char* block = (const char*)src(k, t, seg()) - off + me;
            d += me;
            if (seg_n() > 0 && t >= A.ends && t + A.ends < (unsigned)A.T) {
              for (int b = me; b < bytes; b += step_b, block += step_b, d += step_b)
                copy_async(d, block);
            } else if (seg_n() > 0) {
              for (int b = me; b < bytes; b += step_b, block += step_b, d += step_b) {
                if (block >= (const char*)A.in[k]) {
                  // nothing is read behind the array's last element
                  copy_async(d, block, (uint32_t)min((int64_t)16, (int64_t)((const char*)src(k, A.T - 1, A.H) - block)));
                } else {  // nor before its first
                  for (int j = 0; j < 16; j += sizeof(T))
                    if (b + j >= off && b + j < bytes) *(T*)(d + j) = *(const T*)(block + j);
                }
              }
            }
          } else {
            const T* p = src(k, t, col0);
#pragma unroll
            for (int c = 0; c < NCH; ++c)
              if (c < count) copy_async(d + c * blockDim.x * 16, p + c * size * VEC);
          }
        }
    copy_commit();
  }
  // zeroes the slots of the pieces outside the row and starts the copies of the first
  // rows; then, each round: those of the row stages - 1 rounds ahead, and a wait for
  // this round's
  __device__ void begin() const {
    if constexpr (RING) {
      for (int s = 0; s < A.stages; ++s) {
        if constexpr (!BLOCK) {
#pragma unroll
          for (int k = 0; k < N_IN; ++k)
            if (A.in[k])
#pragma unroll
              for (int c = 0; c < NCH; ++c)
                if (c >= count)
                  *(uint4*)(place(s * A.stage_bytes, k) + c * blockDim.x * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        if (s < A.stages - 1) fetch(s * A.stage_bytes, (unsigned)row + (unsigned)s * step);
      }
    }
  }
  __device__ void advance(unsigned t) const {
    if constexpr (RING) {
      if constexpr (BLOCK) __syncwarp();  // the others have read the stage that is filled now
      fetch(at == 0 ? (A.stages - 1) * A.stage_bytes : at - A.stage_bytes, t + (unsigned)(A.stages - 1) * step);
      if (A.stages == 3) copy_wait<2>();
      else copy_wait<1>();
      if constexpr (BLOCK) __syncwarp();  // what the others copied is here
    }
  }
  __device__ void next() { at = at + A.stage_bytes == A.stages * A.stage_bytes ? 0 : at + A.stage_bytes; }
  // the pieces of array k of row t, zero outside the row: all, or half h of them
  __device__ void read(int k, unsigned t, float2* v) const {
    read_half(k, t, v, 0);
    read_half(k, t, v + N2 / 2, 1);
  }
  __device__ void read_half(int k, unsigned t, float2* v, int h) const {
    const T* g;
    int step_c = apart();
    if constexpr (BLOCK) {
      g = (const T*)(place(at, k) + shift(k, t)) + lane % members();
    } else if constexpr (RING) {
      g = (const T*)place(at, k);
      step_c = blockDim.x * VEC;
    } else {
      g = src(k, t, col0);
    }
#pragma unroll
    for (int c = 0; c < NCH / 2; ++c) {
      const int d = h * (NCH / 2) + c;
      const bool on = (RING && !BLOCK) || (d < count && t < (unsigned)A.T);
      const T* p = g + d * step_c;
      if constexpr (VEC > 1) {
        const uint4 w = on ? *(const uint4*)p : make_uint4(0u, 0u, 0u, 0u);
        if constexpr (sizeof(T) == 4) {
          v[2 * c] = make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
          v[2 * c + 1] = make_float2(__uint_as_float(w.z), __uint_as_float(w.w));
        } else {
          v[4 * c] = bf2(w.x);
          v[4 * c + 1] = bf2(w.y);
          v[4 * c + 2] = bf2(w.z);
          v[4 * c + 3] = bf2(w.w);
        }
      } else {
        const float x = on ? to_f32(*p) : 0.f;
        if (c & 1) v[c / 2].y = x;
        else v[c / 2].x = x;
      }
    }
    if (GRP == WARP && RING && !BLOCK && t >= (unsigned)A.T)  // what an earlier row left
#pragma unroll
      for (int i = 0; i < N2 / 2; ++i) v[i] = make_float2(0.f, 0.f);
  }
  __device__ void write(void* out, unsigned t, const float2* v) const {
    write_half(out, t, v, 0);
    write_half(out, t, v + N2 / 2, 1);
  }
  __device__ void write_half(void* out, unsigned t, const float2* v, int h) const {
    if (GRP == WARP && t >= (unsigned)A.T) return;
    T* g = (T*)out + (uint64_t)t * (unsigned)A.H + col0;
#pragma unroll
    for (int c = 0; c < NCH / 2; ++c)
      if (h * (NCH / 2) + c < count) {
        T* p = BLOCK ? g + (h * (NCH / 2) + c) * members() : g + (h * (NCH / 2) + c) * size * VEC;
        if constexpr (VEC > 1) {
          uint4 w;
          if constexpr (sizeof(T) == 4)
            w = make_uint4(__float_as_uint(v[2 * c].x), __float_as_uint(v[2 * c].y), __float_as_uint(v[2 * c + 1].x),
                           __float_as_uint(v[2 * c + 1].y));
          else
            w = make_uint4(to_bf2(v[4 * c]), to_bf2(v[4 * c + 1]), to_bf2(v[4 * c + 2]), to_bf2(v[4 * c + 3]));
          *(uint4*)p = w;
        } else {
          *p = from_f32<T>(c & 1 ? v[c / 2].y : v[c / 2].x);
        }
      }
  }
  // the row in 8 bits, a piece at a time
  __device__ void write_q8(unsigned t, const float2* v) const {
    if (GRP == WARP && t >= (unsigned)A.T) return;
    uint8_t* g = (uint8_t*)A.q_out + (uint64_t)t * (unsigned)A.H;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
      if (c < count) {
        uint8_t* p = g + col(c);
        if constexpr (VEC == 8)
          *(uint2*)p = make_uint2(to_e4m3(v[4 * c], v[4 * c + 1]), to_e4m3(v[4 * c + 2], v[4 * c + 3]));
        else if constexpr (VEC == 4)
          *(uint32_t*)p = to_e4m3(v[2 * c], v[2 * c + 1]);
        else
          *p = (uint8_t)(to_e4m3(v[c / 2], v[c / 2]) >> (c & 1 ? 8 : 0));
      }
  }
  // element j of piece c in a thread's pairs
  static __device__ float& elem(float2* v, int c, int j) {
    float2& p = v[(c * VEC + j) / 2];
    return (c * VEC + j) & 1 ? p.y : p.x;
  }
  // fp32 parameters of the thread's columns, `rest` where absent
  __device__ void params(const float* p, float add, float rest, float2* v) const {
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int j = 0; j < VEC; ++j) elem(v, c, j) = p && c < count ? add + p[col(c) + j] : rest;
  }
  // sum of the threads' v and largest of their m (bits of what has no sign: a NaN is above
  // infinity) in one exchange, in a buffer of two values
  __device__ void sum_most(float& v, uint32_t& m, float (*buf)[2][COLS][MAX_W], int& turn) const {
    if constexpr (GRP == WARP) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        if (o < size) {
          v += __shfl_xor_sync(0xffffffffu, v, o);
          m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        }
      return;
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    float(*b)[COLS][MAX_W] = buf[turn];
    turn ^= 1;
    v = warp_sum(v);
    m = __reduce_max_sync(0xffffffffu, m);
    int cols = 1;
    if constexpr (GRP == CTA) {
      if (lane == 0) b[0][0][warp] = v, b[1][0][warp] = __uint_as_float(m);
      __syncthreads();
    } else {
      cooperative_groups::cluster_group cl = cooperative_groups::this_cluster();
      cols = cl.num_blocks();
      const int i = lane & 1, c = lane >> 1;
      if (c < cols) *cl.map_shared_rank(&b[i][cl.block_rank()][warp], c) = i ? __uint_as_float(m) : v;
      cl.sync();
    }
    v = 0.f;
    for (int c = 0; c < cols; ++c)
#pragma unroll
      for (int w = 0; w < MAX_W; w += 4)
        if (w < nw) {
          const float4 p = *(const float4*)&b[0][c][w];
          const uint4 q = *(const uint4*)&b[1][c][w];
          v += (p.x + p.y) + (p.z + p.w);
          m = max(max(m, max(q.x, q.y)), max(q.z, q.w));
        }
  }
  // sums of N (1 or 3) values over the row's threads, the same in each of them; buf is
  // used in turn: a half is written again only after the barrier that follows its last
  // reads
  template <int N, int M>
  __device__ void sum(float (&v)[N], float (*buf)[M][COLS][MAX_W], int& turn) const {
    static_assert(N <= M, "a place for every value");
    if constexpr (GRP == WARP) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        if (o < size)
#pragma unroll
          for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
      return;
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    float(*b)[COLS][MAX_W] = buf[turn];
    turn ^= 1;
    float u;
    if constexpr (N == 1) {
      u = warp_sum(v[0]);
    } else {
      // three sums in six exchanges: value i ends in the lanes with lane % 4 == i
      const bool o1 = lane & 1, o2 = lane & 2;
      float p = o1 ? v[1] : v[0], q = o1 ? 0.f : v[2];
      p += __shfl_xor_sync(0xffffffffu, o1 ? v[0] : v[1], 1);
      q += __shfl_xor_sync(0xffffffffu, o1 ? v[2] : 0.f, 1);
      u = o2 ? q : p;
      u += __shfl_xor_sync(0xffffffffu, o2 ? p : q, 2);
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) u += __shfl_xor_sync(0xffffffffu, u, o);
    }
    int cols = 1;
    if constexpr (GRP == CTA) {
      if (lane < N) b[lane][0][warp] = u;
      __syncthreads();
    } else {  // every CTA of the cluster gets every warp's sums
      cooperative_groups::cluster_group cl = cooperative_groups::this_cluster();
      cols = cl.num_blocks();
      const int i = lane & 3, c = lane >> 2;
      if (i < N && c < cols) *cl.map_shared_rank(&b[i][cl.block_rank()][warp], c) = u;
      cl.sync();
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
    for (int c = 0; c < cols; ++c)
#pragma unroll
      for (int w = 0; w < MAX_W; w += 4)
        if (w < nw)
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float4 p = *(const float4*)&b[i][c][w];
            v[i] += (p.x + p.y) + (p.z + p.w);
          }
  }
};

// the places of warps that a CTA does not have stay zero
template <int N, int C, int W>
__device__ __forceinline__ void clear(float (*buf)[N][C][W]) {
  for (int i = threadIdx.x; i < 2 * N * C * W; i += blockDim.x) (&buf[0][0][0][0])[i] = 0.f;
  __syncthreads();
}

extern __shared__ uint4 norm_ring[];

// Q8: h in e4m3 with a scale for each token, its largest magnitude over e4m3's (so that no
// value is cut off), and not below the smallest normal fp32 (a row of zeros).  The row is in
// registers, so the second sweep over it costs a reduction more and no bytes.
template <typename T, int VEC, int GRP, bool Q8>
__global__ void __launch_bounds__(max_threads(GRP), 65536 / REGS / max_threads(GRP))
k_resnorm_fwd(const __grid_constant__ NormArgs A) {
  constexpr int NB = Q8 ? 2 : 1;
  __shared__ __align__(16) float buf[2][NB][max_cols(GRP)][max_threads(GRP) / 32];
  int turn = 0;
  if (GRP == CTA) clear(buf);
  Rows<T, VEC, GRP> R(A, (char*)norm_ring);
  R.begin();
  if constexpr (GRP >= CLUSTER) cooperative_groups::this_cluster().sync();  // all have started
  const float inv = 1.f / (float)A.H;
  const float2 a2 = both(A.a);
  const bool has_y = A.in[IN_Y], post = A.w_post, token = A.gate_kind == LX_GATE_TOKEN;
  float2 w1[N2], w2[N2];  // w1: with the channel gate
  R.params(A.w_post, A.off, 1.f, w1);
  R.params(A.w_pre, A.off, 0.f, w2);
  if (A.gate_kind == LX_GATE_CHANNEL) {
    float2 g[N2];
    R.params(A.gate, 0.f, 0.f, g);
#pragma unroll
    for (int i = 0; i < N2; ++i) w1[i] = muls(w1[i], g[i]);
  }
  // a row's gate is read a round ahead
  float next = token && R.row < A.T ? A.gate[R.row * A.ldg] : 1.f;
  for (unsigned t = R.row; R.more(t); t += R.step, R.next()) {
    const float tok = next;
    if (token && t + R.step < (unsigned)A.T) next = A.gate[(long)(t + R.step) * A.ldg];
    R.advance(t);
    float2 x[N2];
    R.read(IN_R, t, x);
#pragma unroll
    for (int i = 0; i < N2; ++i) x[i] = muls(x[i], a2);
    float s1 = 1.f, s2 = 1.f, q[1];
    if (has_y) {
      float2 y[N2];
      R.read(IN_Y, t, y);
      if (post) {
        float2 p = muls(y[0], y[0]);
#pragma unroll
        for (int i = 1; i < N2; ++i) p = fmas(y[i], y[i], p);
        q[0] = p.x + p.y;
        R.sum(q, buf, turn);
        s1 = rsqrtf(q[0] * inv + A.eps);
      }
      if (A.in[IN_GATE]) {
        float2 g[N2];
        R.read(IN_GATE, t, g);
#pragma unroll
        for (int i = 0; i < N2; ++i) y[i] = muls(y[i], g[i]);
      }
      const float2 f = both(s1 * tok);
#pragma unroll
      for (int i = 0; i < N2; ++i) x[i] = fmas(muls(y[i], w1[i]), f, x[i]);
    }
    if (A.r_out) R.write(A.r_out, t, x);
    if (A.w_pre) {
      float2 p = muls(x[0], x[0]);
#pragma unroll
      for (int i = 1; i < N2; ++i) p = fmas(x[i], x[i], p);
      q[0] = p.x + p.y;
      if constexpr (Q8) {
        // the row's largest |r' w2| with its sum of squares: h is that times s2
        float2 v[N2];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < N2; ++i) {
          v[i] = muls(x[i], w2[i]);
          m = max(m, max(__float_as_uint(v[i].x) & 0x7fffffffu, __float_as_uint(v[i].y) & 0x7fffffffu));
        }
        R.sum_most(q[0], m, buf, turn);
        s2 = rsqrtf(q[0] * inv + A.eps);
        if (A.h_out) {
#pragma unroll
          for (int i = 0; i < N2; ++i) x[i] = muls(muls(x[i], both(s2)), w2[i]);
          R.write(A.h_out, t, x);
        }
        const float top = s2 * __uint_as_float(m);
        const float scale = top < E4M3_MAX * TINY ? TINY : top / E4M3_MAX;
        float by = s2 / scale;  // at most 448 over the row's largest,
        if (__uint_as_float(m) < SMALL) {  // which is above fp32's range below 1.4e-36: its factors one by one
          by = 1.f / scale;
#pragma unroll
          for (int i = 0; i < N2; ++i) v[i] = muls(v[i], both(s2));
        }
#pragma unroll
        for (int i = 0; i < N2; ++i) v[i] = muls(v[i], both(by));
        R.write_q8(t, v);
        if (R.writer() && t < (unsigned)A.T) A.scale[t] = scale;
      } else {
        R.sum(q, buf, turn);
        s2 = rsqrtf(q[0] * inv + A.eps);
#pragma unroll
        for (int i = 0; i < N2; ++i) x[i] = muls(muls(x[i], both(s2)), w2[i]);
        R.write(A.h_out, t, x);
      }
    }
    if (A.stats && R.writer() && t < (unsigned)A.T) {
      A.stats[t] = s1;
      A.stats[(long)A.T + t] = s2;
    }
  }
  // a CTA's shared memory outlives its neighbours' writes
  if constexpr (GRP >= CLUSTER) cooperative_groups::this_cluster().sync();
}

// In the thread's terms, with X = r' = a r + s1 Y, Y = y g W1, E = s2 dh W2, D0 = dr' + E:
// one set of sums, q0 = sum(E X), q1 = sum(D0 Y), q2 = sum(X Y), serves both norms:
//   M = s2^2 q0 / H,  D = D0 - M X,  V = sum(D Y) = q1 - M q2,
//   dy = s1 (D g W1) - s1^3 V / H y        (sum(f n) = s1 V)
// A token's gate is left out of Y (its gradient is s1 V) and put to s1 instead.  A column's
// sum B of s1 D y (with a full or token gate: of s1 g D y) gives dw_post = g B and a channel
// gate's gradient W1 B.
template <typename T, int VEC, int GRP>
__global__ void __launch_bounds__(max_threads(GRP), 65536 / REGS / max_threads(GRP))
k_resnorm_bwd(const __grid_constant__ NormArgs A) {
  __shared__ __align__(16) float buf[2][3][max_cols(GRP)][max_threads(GRP) / 32];
  int turn = 0;
  if (GRP == CTA) clear(buf);
  Rows<T, VEC, GRP> R(A, (char*)norm_ring);
  R.begin();
  if constexpr (GRP >= CLUSTER) cooperative_groups::this_cluster().sync();  // all have started
  const float inv = 1.f / (float)A.H;
  const bool has_y = A.in[IN_Y], post = A.w_post, token = A.gate_kind == LX_GATE_TOKEN, full = A.in[IN_GATE];
  const float2 zero = make_float2(0.f, 0.f);
  constexpr int H2 = N2 / 2;
  // the columns' parameters g W1 (W1 with a full gate) and W2, in slots that only this
  // thread reads: registers are short
  float4* par = (float4*)((char*)norm_ring + A.par_at) + threadIdx.x;
  auto put = [&](int k, const float2* v) {
#pragma unroll
    for (int i = 0; i < N2; i += 2)
      par[(k * (EPT / 4) + i / 2) * blockDim.x] = make_float4(v[i].x, v[i].y, v[i + 1].x, v[i + 1].y);
  };
  auto get = [&](int k, float2* v, int h) {  // half h of them
#pragma unroll
    for (int i = 0; i < H2; i += 2) {
      const float4 p = par[(k * (EPT / 4) + h * (EPT / 8) + i / 2) * blockDim.x];
      v[i] = make_float2(p.x, p.y);
      v[i + 1] = make_float2(p.z, p.w);
    }
  };
  {
    float2 v[N2], g[N2];
    R.params(A.w_post, A.off, 1.f, v);
    R.params(A.gate_kind == LX_GATE_CHANNEL ? A.gate : nullptr, 0.f, 1.f, g);
#pragma unroll
    for (int i = 0; i < N2; ++i) v[i] = mul2(v[i], g[i]);
    put(0, v);
    R.params(A.w_pre, A.off, 0.f, v);
    put(1, v);
  }
  // this launch started after its predecessors had ended: the next may be scheduled
  if (A.part) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  float2 acc[2][N2];  // B, dw_pre
#pragma unroll
  for (int i = 0; i < N2; ++i) acc[0][i] = acc[1][i] = zero;
  float n1 = 0.f, n2 = 0.f, ng = 1.f;  // a row's scalars are read a round ahead
  auto scalars = [&](unsigned t) {
    if (t >= (unsigned)A.T) return;
    n1 = A.stats[t];
    n2 = A.stats[(long)A.T + t];
    if (token) ng = A.gate[(long)t * A.ldg];
  };
  scalars(R.row);
  for (unsigned t = R.row; R.more(t); t += R.step, R.next()) {
    const float s1 = n1, s2 = n2, sg = n1 * ng;  // sg: with the token's gate
    scalars(t + R.step);
    R.advance(t);
    // by halves, so that few values wait; y and Y are formed before and after the sums
    float2 D[N2], X[N2], q0 = zero, q1 = zero, q2 = zero;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float2 Y[H2], *Dh = D + h * H2, *Xh = X + h * H2;
      if (A.in[IN_DR]) R.read_half(IN_DR, t, Dh, h);
      else
#pragma unroll
        for (int i = 0; i < H2; ++i) Dh[i] = zero;
      if (has_y) {
        float2 w[H2];
        get(0, w, h);
        R.read_half(IN_Y, t, Y, h);
#pragma unroll
        for (int i = 0; i < H2; ++i) Y[i] = mul2(Y[i], w[i]);
        if (full) {
          R.read_half(IN_GATE, t, w, h);
#pragma unroll
          for (int i = 0; i < H2; ++i) Y[i] = mul2(Y[i], w[i]);
        }
      }
      if (A.in[IN_DH]) {
        float2 dh[H2], w2[H2];
        get(1, w2, h);
        R.read_half(IN_R, t, Xh, h);
        R.read_half(IN_DH, t, dh, h);
#pragma unroll
        for (int i = 0; i < H2; ++i) {
          Xh[i] = mul2(Xh[i], both(A.a));
          if (has_y) Xh[i] = fma2(both(sg), Y[i], Xh[i]);
          dh[i] = mul2(dh[i], both(s2));
          acc[1][h * H2 + i] = fma2(dh[i], Xh[i], acc[1][h * H2 + i]);
          const float2 E = mul2(dh[i], w2[i]);
          q0 = fma2(E, Xh[i], q0);
          Dh[i] = add2(Dh[i], E);
        }
      } else {
#pragma unroll
        for (int i = 0; i < H2; ++i) Xh[i] = zero;
      }
      if (has_y)
#pragma unroll
        for (int i = 0; i < H2; ++i) {
          q1 = fma2(Dh[i], Y[i], q1);
          q2 = fma2(Xh[i], Y[i], q2);
        }
    }
    float q[3] = {q0.x + q0.y, q1.x + q1.y, q2.x + q2.y};
    R.sum(q, buf, turn);
    const float M = q[0] * inv * s2 * s2;
    const float V = q[1] - M * q[2];
    const float m1 = post ? sg * s1 * s1 * inv * V : 0.f;
    if (token && A.dgate && R.writer() && t < (unsigned)A.T) ((float*)A.dgate)[t] = s1 * V;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float2 *Dh = D + h * H2, *Xh = X + h * H2;
#pragma unroll
      for (int i = 0; i < H2; ++i) {
        Dh[i] = fma2(both(-M), Xh[i], Dh[i]);
        Xh[i] = mul2(Dh[i], both(A.a));
      }
      if (A.dr) R.write_half(A.dr, t, Xh, h);
      if (has_y) {
        float2 y[H2], w[H2];
        R.read_half(IN_Y, t, y, h);
        get(0, w, h);
        if (full) {
          float2 g[H2];
          R.read_half(IN_GATE, t, g, h);
          if (A.dgate) {
#pragma unroll
            for (int i = 0; i < H2; ++i) Xh[i] = mul2(mul2(Dh[i], y[i]), mul2(w[i], both(s1)));
            R.write_half(A.dgate, t, Xh, h);
          }
#pragma unroll
          for (int i = 0; i < H2; ++i) Dh[i] = mul2(Dh[i], g[i]);
        }
#pragma unroll
        for (int i = 0; i < H2; ++i) {
          acc[0][h * H2 + i] = fma2(mul2(Dh[i], y[i]), both(sg), acc[0][h * H2 + i]);
          Dh[i] = fma2(both(-m1), y[i], mul2(mul2(Dh[i], w[i]), both(sg)));
        }
        if (A.dy) R.write_half(A.dy, t, Dh, h);
      }
    }
  }
  if (A.part) {
    float* part = A.part + (GRP >= CLUSTER ? (long)blockIdx.y : (long)blockIdx.x) * 2 * A.H;
    float* ws = (float*)norm_ring;  // [rows of the CTA][H], the slots' copies being done
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (!(A.sums >> k & 1)) continue;
      if constexpr (GRP == WARP) {
        copy_wait<0>();
        __syncthreads();
#pragma unroll
        for (int c = 0; c < R.NCH; ++c)
          if (c < R.count)
#pragma unroll
            for (int j = 0; j < VEC; ++j) ws[(threadIdx.x / R.size) * A.H + R.col(c) + j] = R.elem(acc[k], c, j);
        __syncthreads();
        for (int e = threadIdx.x; e < A.H; e += CTA_T) {
          float s = 0.f;
          for (int w = 0; w < CTA_T / R.size; ++w) s += ws[w * A.H + e];
          part[(long)k * A.H + e] = s;
        }
      } else {
#pragma unroll
        for (int c = 0; c < R.NCH; ++c)
          if (c < R.count)
#pragma unroll
            for (int j = 0; j < VEC; ++j) part[(long)k * A.H + R.col(c) + j] = R.elem(acc[k], c, j);
      }
    }
  }
  if constexpr (GRP >= CLUSTER) cooperative_groups::this_cluster().sync();
}

// Adds part[p][k][e] over p in a fixed order: 32 columns and 32 ranges of p a CTA; k = 0
// gives dw_post and a channel gate's gradient, 1 dw_pre.  Starts beside the backward's
// last CTAs.
__global__ void __launch_bounds__(1024)
k_resnorm_sum(const __grid_constant__ NormArgs A, int n, float* dw_post, float* dgate, float* dw_pre) {
  __shared__ float sm[32][33];
  const int k = A.sums == 2 ? 1 : blockIdx.y, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int e = blockIdx.x * 32 + lane;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float s = 0.f;
  if (e < A.H)
#pragma unroll 8
    for (int p = w; p < n; p += 32) s += A.part[((long)p * 2 + k) * A.H + e];
  sm[w][lane] = s;
  __syncthreads();
  s = warp_sum(sm[lane][w]);  // column w
  const int c = blockIdx.x * 32 + w;
  if (lane != 0 || c >= A.H) return;
  if (k == 1) {
    dw_pre[c] = s;
  } else {
    if (dw_post) dw_post[c] = A.gate_kind == LX_GATE_CHANNEL ? s * A.gate[c] : s;
    if (dgate) dgate[c] = A.w_post ? s * (A.off + A.w_post[c]) : s;
  }
}

struct Shape {
  int grp, threads, cols, lanes;  // cols: CTAs to a row
  long groups;                    // CTAs (clusters) that have a row
};

Shape shape_of(int T, int H) {
  Shape s;
  s.grp = H <= WARP_H ? WARP : H <= CTA_T * EPT ? CTA : H <= CTA_T * EPT * MAX_CLUSTER ? CLUSTER : WIDE;
  s.threads = s.grp == CTA ? (H + 32 * EPT - 1) / (32 * EPT) * 32 : max_threads(s.grp);
  s.cols = s.grp >= CLUSTER ? (H + s.threads * EPT - 1) / (s.threads * EPT) : 1;
  s.lanes = 4;  // (a group's slots have a block more than its columns)
  while (s.lanes < 32 && s.lanes * EPT < H) s.lanes *= 2;
  const int rows = s.grp == WARP ? CTA_T / s.lanes : 1;
  s.groups = ((long)T + rows - 1) / rows;
  return s;
}

// CTAs (clusters) that rows are dealt to: as many as the SMs hold, by their registers
// (this bounds the backward's workspace) and with `smem` bytes each
int ctas_per_sm(const Shape& s) { return std::max(1, 65536 / (REGS * s.threads)); }
int resident(const Shape& s, size_t smem) {
  const long ctas = std::min<long>(ctas_per_sm(s), std::max<long>(1, 227 * 1024 / (smem + 2048)));
  return (int)std::min(s.groups, std::max(1L, SMS * ctas / s.cols));
}

// Slots of a CTA: three rows, or two where three would not fit beside the SM's other CTAs
size_t ring_bytes(const Shape& s, NormArgs& A, size_t es, size_t more, bool block) {
  const int members = s.grp == WARP ? s.lanes : 32;
  size_t row = 0;
  A.ends = 1;
  for (int k = 0; k < N_IN; ++k)
    if (A.in[k]) {
      A.ends = std::max(A.ends, end_rows(A.ldb[k]));
      A.slot_at[k] = (uint32_t)row;
      row += block ? (size_t)(s.threads / members) * group_bytes(members, es) : EPT * es * s.threads;
    }
  A.stage_bytes = (uint32_t)row;
  A.stages = (3 * row + more + 1024) * ctas_per_sm(s) <= 227 * 1024 ? 3 : 2;
  return A.stages * row;
}

template <typename... KArgs>
lx_status launch(void (*kern)(KArgs...), const Shape& s, int groups, size_t smem, const NormArgs& A, cudaStream_t st,
                 bool (&cap)[64]) {
  int dev = 0;
  LX_CUDA(cudaGetDevice(&dev));
  LX_CUDA(smem_cap_once((const void*)kern, 224 * 1024, dev, cap));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = s.grp >= CLUSTER ? dim3(s.cols, (unsigned)groups) : dim3((unsigned)groups);
  cfg.blockDim = dim3(s.threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = s.cols;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = s.grp >= CLUSTER ? 1 : 0;
  LX_CUDA(cudaLaunchKernelEx(&cfg, kern, A));
  return LX_OK;
}

enum Kind { FWD = 0, FWD_Q8 = 1, BACKWARD = 2 };

template <typename T, int VEC, int GRP, int KIND>
lx_status launch_one(const Shape& s, NormArgs& A, cudaStream_t st, int& groups) {
  static bool cap[64] = {};
  constexpr bool BWD = KIND == BACKWARD;
  const size_t par = BWD ? sizeof(float) * 2 * EPT * s.threads : 0;
  size_t smem = 0;
  A.stages = 2;
  if (Rows<T, VEC, GRP>::RING) smem = ring_bytes(s, A, sizeof(T), par, Rows<T, VEC, GRP>::BLOCK);
  A.par_at = (uint32_t)smem;  // (a multiple of 16)
  smem += par;
  if (BWD && GRP == WARP) smem = std::max(smem, sizeof(float) * (CTA_T / s.lanes) * A.H);
  groups = resident(s, smem);
  // A backward of few rows: a CTA an SM (two where rows are copied in blocks) as long as that
  // leaves a CTA under 7 rows: every CTA more writes column sums as large as a row (2048
  // bf16: 300 rows 11.2 us with 152 CTAs, 13.4 with 304; 1031 rows 17.0, 16.5, 21.8 with 608;
  // 4000 of 2560: 44.8, 33.6, 34.4; 1031 of 2047: 31.7, 27.2, 27.6).
  using R = Rows<T, VEC, GRP>;
  if (BWD && GRP == CTA && R::RING) groups = std::min(groups, std::max(R::BLOCK ? 2 * SMS : SMS, A.T / 7));
  if constexpr (BWD) return launch(k_resnorm_bwd<T, VEC, GRP>, s, groups, smem, A, st, cap);
  else return launch(k_resnorm_fwd<T, VEC, GRP, KIND == FWD_Q8>, s, groups, smem, A, st, cap);
}

template <typename T, int VEC, int KIND>
lx_status launch_vec(const Shape& s, NormArgs& A, cudaStream_t st, int& groups) {
  if (s.grp == WARP) return launch_one<T, VEC, WARP, KIND>(s, A, st, groups);
  if (s.grp == CTA) return launch_one<T, VEC, CTA, KIND>(s, A, st, groups);
  if (s.grp == CLUSTER) return launch_one<T, VEC, CLUSTER, KIND>(s, A, st, groups);
  return launch_one<T, VEC, WIDE, KIND>(s, A, st, groups);
}

// wide: every row starts on a 16-byte boundary and is a multiple of 16 bytes; groups: out,
// the CTAs (clusters) launched
template <int KIND>
lx_status launch_any(int dtype, bool wide, const Shape& s, NormArgs& A, cudaStream_t st, int& groups) {
  if (dtype == LX_F32)
    return wide ? launch_vec<float, 4, KIND>(s, A, st, groups) : launch_vec<float, 1, KIND>(s, A, st, groups);
  return wide ? launch_vec<__nv_bfloat16, 8, KIND>(s, A, st, groups)
              : launch_vec<__nv_bfloat16, 1, KIND>(s, A, st, groups);
}

constexpr int64_t MAX_LD = (1 << 30) - 1;  // elements between rows: a distance in bytes fits 32 bits
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
  if (d->T > 1 && (d->ldr > MAX_LD || (d->y && d->ldy > MAX_LD) || (d->gate && d->ldg > MAX_LD)))
    return fail(LX_ERR_SHAPE, "rows are 2^30 elements apart or more");
  const size_t es = esize(d->dtype);
  if (!aligned(d->r, es) || !aligned(d->y, es) || !aligned(d->gate, d->gate_kind == LX_GATE_FULL ? es : 4) ||
      !aligned(d->w_post, 4) || !aligned(d->w_pre, 4))
    return fail(LX_ERR_ARG, "a pointer is not aligned to its element");
  return LX_OK;
}

uint32_t row_bytes(const lx_resnorm_desc* d, int64_t ld) { return (uint32_t)(d->T > 1 ? ld * (int64_t)esize(d->dtype) : 0); }

NormArgs args_of(const lx_resnorm_desc* d, const Shape& s) {
  NormArgs A = {};
  A.T = d->T;
  A.H = d->H;
  A.gate_kind = d->gate_kind;
  A.lanes = s.lanes;
  A.in[IN_Y] = d->y;
  A.ldb[IN_Y] = row_bytes(d, d->ldy);
  A.in[IN_R] = d->r;
  A.ldb[IN_R] = row_bytes(d, d->ldr);
  if (d->gate_kind == LX_GATE_FULL) {
    A.in[IN_GATE] = d->gate;
    A.ldb[IN_GATE] = row_bytes(d, d->ldg);
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

bool rows16(const NormArgs& A, size_t es, std::initializer_list<const void*> outs) {
  uintptr_t bits = (uintptr_t)A.H * es;
  for (int k = 0; k < N_IN; ++k)
    if (A.in[k]) bits |= (uintptr_t)A.in[k] | (uintptr_t)A.ldb[k];
  for (const void* p : outs) bits |= (uintptr_t)p;
  return bits % 16 == 0;
}

}  // namespace
}  // namespace lx

namespace lx {
namespace {
// what the two forward calls check alike, with the outputs given and the arguments filled
lx_status forward_args(const lx_resnorm_desc* d, void* r_out, void* h_out, float* stats, const Shape& s, NormArgs& A) {
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
  A = args_of(d, s);
  A.r_out = r_out;
  A.h_out = h_out;
  A.stats = stats;
  return LX_OK;
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
  const Shape s = shape_of(d->T, d->H);
  NormArgs A;
  LX_TRY(forward_args(d, r_out, h_out, stats, s, A));
  int groups;
  return launch_any<FWD>(d->dtype, rows16(A, esize(d->dtype), {r_out, h_out}), s, A, (cudaStream_t)stream, groups);
}

extern "C" lx_status lx_residual_norm_q8(const lx_resnorm_desc* d, void* r_out, void* q_out, float* scale, void* h_out,
                                         float* stats, void* stream) {
  using namespace lx;
  LX_TRY(check_desc(d));
  if (d->T == 0) return LX_OK;
  if (!d->w_pre) return fail(LX_ERR_ARG, "w_pre is NULL");
  if (!q_out || !scale) return fail(LX_ERR_ARG, "q_out or scale is NULL");
  if (!aligned(scale, 4)) return fail(LX_ERR_ARG, "a pointer is not aligned to its element");
  const Shape s = shape_of(d->T, d->H);
  NormArgs A;
  LX_TRY(forward_args(d, r_out, h_out, stats, s, A));
  const size_t es = esize(d->dtype), out = (size_t)d->T * d->H, sc = 4 * (size_t)d->T;
  const void* others[] = {d->r, d->y, d->gate, d->w_post, d->w_pre, r_out, h_out, stats};
  const size_t sizes[] = {span(d->T, d->H, d->ldr, es),
                          span(d->T, d->H, d->ldy, es),
                          d->gate_kind == LX_GATE_FULL    ? span(d->T, d->H, d->ldg, es)
                          : d->gate_kind == LX_GATE_TOKEN ? span(d->T, 1, d->ldg, 4)
                                                          : 4 * (size_t)d->H,
                          4 * (size_t)d->H,
                          4 * (size_t)d->H,
                          out * es,
                          out * es,
                          2 * sc};
  for (int i = 0; i < 8; ++i)
    if (overlap(q_out, out, others[i], sizes[i]) || overlap(scale, sc, others[i], sizes[i]))
      return fail(LX_ERR_ARG, "q_out or scale overlaps another array");
  if (overlap(q_out, out, scale, sc)) return fail(LX_ERR_ARG, "two outputs overlap");
  A.q_out = q_out;
  A.scale = scale;
  int groups;
  return launch_any<FWD_Q8>(d->dtype, rows16(A, es, {r_out, h_out, q_out}), s, A, (cudaStream_t)stream, groups);
}

extern "C" lx_status lx_residual_norm_workspace(int32_t T, int32_t H, uint64_t* bytes) {
  using namespace lx;
  if (!bytes) return fail(LX_ERR_ARG, "bytes is NULL");
  if (T < 0) return fail(LX_ERR_ARG, "T < 0");
  if (H < 1 || H > LX_MAX_WIDTH) return fail(LX_ERR_SHAPE, "H must be in 1..LX_MAX_WIDTH");
  *bytes = (uint64_t)resident(shape_of(T, H), 0) * 2 * H * sizeof(float);
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
  if (d->T > 1 && ((dr_out && lddr > MAX_LD) || (dh && lddh > MAX_LD)))
    return fail(LX_ERR_SHAPE, "rows are 2^30 elements apart or more");
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
  if (params) {
    if (!workspace || !aligned(workspace, 16)) return fail(LX_ERR_ARG, "workspace is NULL or not 16-byte aligned");
    if (workspace_bytes < (uint64_t)resident(s, 0) * 2 * d->H * sizeof(float)) return fail(LX_ERR_ARG, "workspace too small");
  }
  NormArgs A = args_of(d, s);
  if (!dh) A.in[IN_R] = nullptr;  // only the second norm's gradient reads r
  A.stats = const_cast<float*>(stats);
  A.in[IN_DR] = dr_out;
  A.ldb[IN_DR] = row_bytes(d, lddr);
  A.in[IN_DH] = dh;
  A.ldb[IN_DH] = row_bytes(d, lddh);
  A.dr = dr;
  A.dy = dy;
  A.dgate = dgate;
  A.part = params ? (float*)workspace : nullptr;
  A.sums = (dw_post || dgc ? 1 : 0) | (dw_pre ? 2 : 0);
  int groups;
  LX_TRY(launch_any<BACKWARD>(d->dtype, rows16(A, es, {outs[0], outs[1], outs[2]}), s, A, st, groups));
  if (params) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((d->H + 31) / 32, A.sums == 3 ? 2 : 1);
    cfg.blockDim = dim3(1024);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    LX_CUDA(cudaLaunchKernelEx(&cfg, k_resnorm_sum, A, groups, dw_post, dgc, dw_pre));
  }
  return LX_OK;
}
