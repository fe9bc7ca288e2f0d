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
// Both are bound by memory: a row is read once and stays in registers as fp32 (8
// elements a thread), so the forward moves r, y (and a full gate), r' and h, the
// backward r, y, dr', dh, dr and dy; r' is formed again from r and y instead of being
// read, which costs no bytes and keeps the unrounded values.
//
// A row is held by a warp (H <= 256), by a CTA (H <= 8192) or by a cluster of CTAs
// with 8192 columns each.  In the backward, rows are dealt to a resident grid and
// every thread keeps its columns' parameter gradients in registers; the sums of the
// CTAs are added in order by a second launch, so results do not change from run to
// run.
#include <algorithm>

#include "lx_rows.cuh"

namespace lx {
namespace {

using namespace rows;

constexpr int EPT = 8;             // elements of a row a thread holds
constexpr int WARP_H = 32 * EPT;   // widest row of a warp
constexpr int CTA_H = 1024 * EPT;  // widest row of a CTA
constexpr int MAX_CLUSTER = 8;
static_assert(CTA_H * MAX_CLUSTER == LX_MAX_WIDTH, "the widest row");
constexpr int WARP_ROWS = 8;       // rows (warps) of a CTA with a warp to a row

struct NormArgs {
  int T, H, gate_kind;
  long ldr, ldy, ldg, lddr, lddh;
  const void *r, *y, *gate;
  const float *w_post, *w_pre;
  float a, off, eps;
  void *r_out, *h_out;
  float* stats;  // [2][T]: s1, s2
  // backward
  const void *dr_out, *dh;
  void *dr, *dy, *dgate;
  float* part;  // [CTAs of a column range][3][H]: dw_post, dgate (channel), dw_pre
};

enum Group { WARP = 0, CTA = 1, CLUSTER = 2 };

// Which row and which columns a thread works on
template <int GRP>
struct Place {
  int lane, size;  // of the threads that hold a row piece
  int col0;        // first column of the piece
  long row, rows;  // first row, rows between two of this group's rows
  __device__ Place() {
    if constexpr (GRP == WARP) {
      lane = threadIdx.x & 31;
      size = 32;
      col0 = 0;
      row = (long)blockIdx.x * WARP_ROWS + (threadIdx.x >> 5);
      rows = (long)gridDim.x * WARP_ROWS;
    } else {
      lane = threadIdx.x;
      size = blockDim.x;
      col0 = GRP == CTA ? 0 : (int)blockIdx.x * CTA_H;
      row = GRP == CTA ? blockIdx.x : blockIdx.y;
      rows = GRP == CTA ? gridDim.x : gridDim.y;
    }
  }
};

template <int GRP>
__device__ __forceinline__ float row_sum(float v, float (*buf)[32], int& turn) {
  if constexpr (GRP == WARP) return warp_sum(v);
  else return group_sum<GRP == CLUSTER>(v, buf, turn);
}

// Columns of piece c of a thread: from col(c), VEC of them, or none
template <int GRP, int VEC>
__device__ __forceinline__ int col_of(const Place<GRP>& p, int c) {
  return p.col0 + (c * p.size + p.lane) * VEC;
}
template <int GRP>
__device__ __forceinline__ int col_end(const Place<GRP>& p, int H) {
  return GRP == CLUSTER ? min(H, p.col0 + CTA_H) : H;
}

// Gate value of row t, element e
template <typename T, int VEC>
__device__ __forceinline__ void load_gate(const NormArgs& A, long t, int e, float* g) {
  if (A.gate_kind == LX_GATE_FULL) {
    load<T, VEC>((const T*)A.gate + t * A.ldg + e, g);
  } else {
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      g[j] = A.gate_kind == LX_GATE_CHANNEL ? ((const float*)A.gate)[e + j]
             : A.gate_kind == LX_GATE_TOKEN ? ((const float*)A.gate)[t * A.ldg]
                                            : 1.f;
  }
}

template <typename T, int VEC, int GRP>
__global__ void __launch_bounds__(GRP == WARP ? 32 * WARP_ROWS : 1024)
k_resnorm_fwd(const NormArgs A) {
  constexpr int NCH = EPT / VEC;
  __shared__ float buf[2][32];
  int turn = 0;
  const Place<GRP> P;
  const int end = col_end<GRP>(P, A.H);
  const float inv = 1.f / (float)A.H;
  for (long t = P.row; t < A.T; t += P.rows) {
    float x[EPT], y[EPT];
    float s1 = 1.f;
    if (A.y) {
      float q = 0.f;
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int e = col_of<GRP, VEC>(P, c);
#pragma unroll
        for (int j = 0; j < VEC; ++j) y[c * VEC + j] = 0.f;
        if (e < end) load<T, VEC>((const T*)A.y + t * A.ldy + e, y + c * VEC);
#pragma unroll
        for (int j = 0; j < VEC; ++j) q = fmaf(y[c * VEC + j], y[c * VEC + j], q);
      }
      if (A.w_post) s1 = rsqrtf(row_sum<GRP>(q, buf, turn) * inv + A.eps);
    }
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e = col_of<GRP, VEC>(P, c);
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[c * VEC + j] = 0.f;
      if (e < end) {
        load<T, VEC>((const T*)A.r + t * A.ldr + e, x + c * VEC);
        float g[VEC];
        if (A.y) load_gate<T, VEC>(A, t, e, g);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          float v = A.a * x[c * VEC + j];
          if (A.y) {
            float u = y[c * VEC + j];
            if (A.w_post) u *= s1 * (A.off + A.w_post[e + j]);
            v = fmaf(g[j], u, v);
          }
          x[c * VEC + j] = v;
          q = fmaf(v, v, q);
        }
        if (A.r_out) store<T, VEC>((T*)A.r_out + t * A.H + e, x + c * VEC);
      }
    }
    float s2 = 1.f;
    if (A.w_pre) {
      s2 = rsqrtf(row_sum<GRP>(q, buf, turn) * inv + A.eps);
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int e = col_of<GRP, VEC>(P, c);
        if (e < end) {
          float v[VEC];
#pragma unroll
          for (int j = 0; j < VEC; ++j) v[j] = x[c * VEC + j] * (s2 * (A.off + A.w_pre[e + j]));
          store<T, VEC>((T*)A.h_out + t * A.H + e, v);
        }
      }
    }
    if (A.stats && P.lane == 0 && P.col0 == 0) {
      A.stats[t] = s1;
      A.stats[(long)A.T + t] = s2;
    }
  }
  // a CTA's shared memory outlives its neighbours' reads
  if constexpr (GRP == CLUSTER) cooperative_groups::this_cluster().sync();
}

// Parameter-gradient sums of a thread: its columns of dw_post, the channel gate, dw_pre
template <typename T, int VEC, int GRP>
__global__ void __launch_bounds__(GRP == WARP ? 32 * WARP_ROWS : 1024)
k_resnorm_bwd(const NormArgs A) {
  constexpr int NCH = EPT / VEC;
  __shared__ float buf[2][32];
  __shared__ float wsum[GRP == WARP ? WARP_ROWS : 1][GRP == WARP ? WARP_H : 1];
  int turn = 0;
  const Place<GRP> P;
  const int end = col_end<GRP>(P, A.H);
  const float inv = 1.f / (float)A.H;
  float acc[3][EPT];
#pragma unroll
  for (int i = 0; i < EPT; ++i) acc[0][i] = acc[1][i] = acc[2][i] = 0.f;
  for (long t = P.row; t < A.T; t += P.rows) {
    const float s1 = A.stats[t], s2 = A.stats[(long)A.T + t];
    float n[EPT], D[EPT], x[EPT], g[EPT];  // n: y s1 (or y)
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e = col_of<GRP, VEC>(P, c);
#pragma unroll
      for (int j = 0; j < VEC; ++j) n[c * VEC + j] = D[c * VEC + j] = x[c * VEC + j] = g[c * VEC + j] = 0.f;
      if (e < end) {
        if (A.y) {
          load<T, VEC>((const T*)A.y + t * A.ldy + e, n + c * VEC);
          load_gate<T, VEC>(A, t, e, g + c * VEC);
        }
        if (A.dr_out) load<T, VEC>((const T*)A.dr_out + t * A.lddr + e, D + c * VEC);
        if (A.dh) {
          float dh[VEC];
          load<T, VEC>((const T*)A.dh + t * A.lddh + e, dh);
          load<T, VEC>((const T*)A.r + t * A.ldr + e, x + c * VEC);
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const int i = c * VEC + j;
            float v = A.a * x[i];
            if (A.y) {
              float u = n[i];
              if (A.w_post) u *= s1 * (A.off + A.w_post[e + j]);
              v = fmaf(g[i], u, v);
            }
            x[i] = v * s2;
            acc[2][i] = fmaf(dh[j], x[i], acc[2][i]);
            const float ev = dh[j] * (A.off + A.w_pre[e + j]);
            q = fmaf(ev, x[i], q);
            D[i] = fmaf(s2, ev, D[i]);
          }
        }
      }
    }
    if (A.dh) {
      const float m = row_sum<GRP>(q, buf, turn) * inv * s2;
#pragma unroll
      for (int i = 0; i < EPT; ++i) D[i] = fmaf(-m, x[i], D[i]);
    }
    float q1 = 0.f, q2 = 0.f;  // f n and D u
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e = col_of<GRP, VEC>(P, c);
      if (e < end) {
        float v[VEC];
        if (A.dr) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) v[j] = A.a * D[c * VEC + j];
          store<T, VEC>((T*)A.dr + t * A.H + e, v);
        }
        if (A.y) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const int i = c * VEC + j;
            const float w = A.w_post ? A.off + A.w_post[e + j] : 1.f;
            n[i] *= s1;
            const float du = D[i] * (n[i] * w);
            q2 += du;
            acc[1][i] += du;
            v[j] = du;
            const float f = g[i] * D[i];
            acc[0][i] = fmaf(f, n[i], acc[0][i]);
            D[i] = f * w;
            q1 = fmaf(D[i], n[i], q1);
          }
          if (A.gate_kind == LX_GATE_FULL && A.dgate) store<T, VEC>((T*)A.dgate + t * A.H + e, v);
        }
      }
    }
    if (A.y) {
      float m = 0.f;
      if (A.w_post) m = row_sum<GRP>(q1, buf, turn) * inv;
      if (A.gate_kind == LX_GATE_TOKEN && A.dgate) {
        const float d = row_sum<GRP>(q2, buf, turn);
        if (P.lane == 0 && P.col0 == 0) ((float*)A.dgate)[t] = d;
      }
      if (A.dy) {
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
          const int e = col_of<GRP, VEC>(P, c);
          if (e < end) {
            float v[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[j] = s1 * fmaf(-m, n[c * VEC + j], D[c * VEC + j]);
            store<T, VEC>((T*)A.dy + t * A.H + e, v);
          }
        }
      }
    }
  }
  if (A.part) {
    float* part = A.part + (GRP == CLUSTER ? (long)blockIdx.y : (long)blockIdx.x) * 3 * A.H;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      if constexpr (GRP == WARP) {
        __syncthreads();
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            wsum[threadIdx.x >> 5][col_of<GRP, VEC>(P, c) + j] = acc[k][c * VEC + j];
        __syncthreads();
        for (int e = threadIdx.x; e < A.H; e += 32 * WARP_ROWS) {
          float s = 0.f;
          for (int w = 0; w < WARP_ROWS; ++w) s += wsum[w][e];
          part[(long)k * A.H + e] = s;
        }
      } else {
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
          const int e = col_of<GRP, VEC>(P, c);
          if (e < end)
#pragma unroll
            for (int j = 0; j < VEC; ++j) part[(long)k * A.H + e + j] = acc[k][c * VEC + j];
        }
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
  int grp, threads, cols;  // cols: CTAs to a row
  long groups;             // rows in work at once with one CTA (or cluster) each
};

Shape shape_of(int T, int H) {
  Shape s;
  s.grp = H <= WARP_H ? WARP : H <= CTA_H ? CTA : CLUSTER;
  s.cols = s.grp == CLUSTER ? (H + CTA_H - 1) / CTA_H : 1;
  s.threads = s.grp == WARP ? 32 * WARP_ROWS : s.grp == CTA ? (((H + EPT - 1) / EPT + 31) / 32) * 32 : 1024;
  s.groups = s.grp == WARP ? ((long)T + WARP_ROWS - 1) / WARP_ROWS : T;
  return s;
}

// CTAs (or clusters) that the backward deals its rows to: two CTAs an SM of the GB300
long bwd_groups(const Shape& s) {
  const long res = s.grp == CLUSTER ? 152 / s.cols : s.grp == WARP ? 152 * 4 : 152 * std::max(1, 1024 / s.threads);
  return std::min(s.groups, std::max(1L, res));
}

template <typename... KArgs>
lx_status launch(void (*kern)(KArgs...), const Shape& s, long groups, const NormArgs& A, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = s.grp == CLUSTER ? dim3(s.cols, (unsigned)groups) : dim3((unsigned)groups);
  cfg.blockDim = dim3(s.threads);
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

template <typename T, bool BWD>
lx_status launch_type(bool vec, const Shape& s, long groups, const NormArgs& A, cudaStream_t st) {
  constexpr int V = 16 / sizeof(T);
#define LX_NORM_CASE(VEC, GRP) \
  return BWD ? launch(k_resnorm_bwd<T, VEC, GRP>, s, groups, A, st) : launch(k_resnorm_fwd<T, VEC, GRP>, s, groups, A, st)
  if (vec) {
    if (s.grp == WARP) LX_NORM_CASE(V, WARP);
    if (s.grp == CTA) LX_NORM_CASE(V, CTA);
    LX_NORM_CASE(V, CLUSTER);
  }
  if (s.grp == WARP) LX_NORM_CASE(1, WARP);
  if (s.grp == CTA) LX_NORM_CASE(1, CTA);
  LX_NORM_CASE(1, CLUSTER);
#undef LX_NORM_CASE
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

NormArgs args_of(const lx_resnorm_desc* d) {
  NormArgs A = {};
  A.T = d->T;
  A.H = d->H;
  A.gate_kind = d->gate_kind;
  A.ldr = d->ldr;
  A.ldy = d->ldy;
  A.ldg = d->ldg;
  A.r = d->r;
  A.y = d->y;
  A.gate = d->gate;
  A.w_post = d->w_post;
  A.w_pre = d->w_pre;
  A.a = d->res_scale;
  A.off = d->weight_offset;
  A.eps = d->eps;
  return A;
}

// whether every row of p starts on a 16-byte boundary
bool rows16(const void* p, long ld, size_t es) { return !p || (aligned(p, 16) && ld * es % 16 == 0); }

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
  NormArgs A = args_of(d);
  A.r_out = r_out;
  A.h_out = h_out;
  A.stats = stats;
  const bool vec = d->H % (16 / es) == 0 && rows16(d->r, d->ldr, es) && rows16(d->y, d->ldy, es) &&
                   (d->gate_kind != LX_GATE_FULL || rows16(d->gate, d->ldg, es)) && aligned(r_out, 16) &&
                   aligned(h_out, 16);
  const Shape s = shape_of(d->T, d->H);
  const long groups = s.grp == CLUSTER ? std::min(s.groups, 65535L) : s.groups;
  cudaStream_t st = (cudaStream_t)stream;
  return d->dtype == LX_BF16 ? launch_type<__nv_bfloat16, false>(vec, s, groups, A, st)
                             : launch_type<float, false>(vec, s, groups, A, st);
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
  bool vec = d->H % (16 / es) == 0;
  for (int i = 0; i < 3; ++i) {
    vec = vec && aligned(outs[i], 16);
    for (int j = 0; j < 5; ++j)
      if (overlap(outs[i], out, ins[j], span(d->T, d->H, lds[j], es)))
        return fail(LX_ERR_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], out, outs[j], out)) return fail(LX_ERR_ARG, "two outputs overlap");
  }
  for (int j = 0; j < 5; ++j) vec = vec && rows16(ins[j], lds[j], es);
  const Shape s = shape_of(d->T, d->H);
  const long groups = bwd_groups(s);
  if (params) {
    if (!workspace || !aligned(workspace, 16)) return fail(LX_ERR_ARG, "workspace is NULL or not 16-byte aligned");
    if (workspace_bytes < (uint64_t)groups * 3 * d->H * sizeof(float)) return fail(LX_ERR_ARG, "workspace too small");
  }
  NormArgs A = args_of(d);
  A.stats = const_cast<float*>(stats);
  A.dr_out = dr_out;
  A.lddr = lddr;
  A.dh = dh;
  A.lddh = lddh;
  A.dr = dr;
  A.dy = dy;
  A.dgate = dgate;
  A.part = params ? (float*)workspace : nullptr;
  LX_TRY(d->dtype == LX_BF16 ? (launch_type<__nv_bfloat16, true>(vec, s, groups, A, st))
                             : (launch_type<float, true>(vec, s, groups, A, st)));
  if (params) {
    k_resnorm_sum<<<dim3((d->H + 31) / 32, 3), 256, 0, st>>>(A.part, (int)groups, d->H, dw_post, dgc, dw_pre);
    LX_CUDA(cudaGetLastError());
  }
  return LX_OK;
}
