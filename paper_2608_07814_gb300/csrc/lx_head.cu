// Softmax cross-entropy over the vocabulary from the last hidden states and the head's
// weights (lx_head_loss), without a [T][V] of logits where that is large:
//   z = h W^T,  loss_t = w_t (log sum_v exp(z_tv) - z_t,label)
//   dz_tv = softmax(z_t)_v - [v = label_t],  dh = w (dz W),  dW = dz^T (w h)
// dz is rounded to bf16 as the tensor cores take it.  The weights stay outside of it: a label's
// entry, which is most of its row, is then about -1 and loses next to nothing.  Blocks of rows are 32 and
// more, so up to 16 tokens have room for w dz in two of them, its value in bf16 and the rest in
// bf16 (2^-16 of it off): their gradients are then rounded once, at the end.  (One token's dW was 1.6 times
// as far off as the plain form's with dz rounded.  Up to 32 tokens, in two blocks: 4 us more.)
// Tokens without a label (or of weight 0) take no part: the others' hidden states are copied
// side by side first, so that they cost no products and what they hold reaches nothing.
// Then (all products on lx_product.cuh):
//   1  the logits' tiles, of which each keeps a row's largest value and sum of exponentials
//      (fp32), 8 bytes for 128 logits, and one of them the label's logit;
//   2  each row's log-sum-exp and loss, (largest - label's) + log of the sum: what a sure row's
//      is made of is not the difference of two large numbers, and no loss is below 0;
//   3  by pieces of the vocabulary: the logits again, now turned into dz (bf16) on their way out
//      of the tensor core, and the two gradient products of the piece in one launch.  dh is
//      held in fp32 between the pieces.
// With the logits formed twice that is 8 T V H operations against the 6 that a kept [T][V]
// needs, and a workspace that grows with T V by those 8 bytes alone.  The label's dz comes from step
// 2 as well, from its loss.  Where all logits fit, as fp32, into the room of a piece, they are kept
// in a room of their own and step 3 reads them instead of W: few tokens would spend as long on reading
// W again as on everything else.
#include "lx_product.cuh"

namespace lx {
namespace {

using namespace rows;
using namespace prod;

constexpr int ROWS = 8;                      // of a CTA of k_head_rows, one a warp
constexpr int RUN = 2048;                    // rows that k_head_rows counts by itself
constexpr int FEW = 16;                      // tokens whose dz is held in two rows, FEW apart
constexpr long PIECE_BYTES = 256L << 20;     // of dz, or of kept logits, at most
constexpr int MAX_T = 1 << 24, MAX_V = 1 << 24, MAX_H = 1 << 20;

struct Head {
  int T, V, H, Tp;  // Tp: rows of the compact arrays, a multiple of 256
  const __nv_bfloat16* h;
  long ldh;
  const int* labels;
  const float* row_weight;
  float* loss;
  __nv_bfloat16* dh;
  // compact
  __nv_bfloat16 *hc, *hw;  // hidden states, and those times the weights (hc itself without weights,
  bool few;                // and with up to FEW tokens, whose rows it has twice)
  int *label, *row, *n;
  int* runs;  // rows that count of each RUN, where there are more
  float *weight, *lse2;
  float* own;           // the label's logit, then its dz
  const float2* part;
  int slots;
  const float* keep;    // the logits, keep_cols blocks side by side
  int keep_cols;
  __nv_bfloat16* dl;
  long ldd;
};

__device__ __forceinline__ int counts(const Head& A, int t) {
  const int l = A.labels[t];
  const float w = A.row_weight ? A.row_weight[t] : 1.f;
  return l >= 0 && l < A.V && w != 0.f;
}

// rows that count of each RUN
__global__ void __launch_bounds__(256) k_head_runs(const __grid_constant__ Head A) {
  __shared__ int red[8];
  pdl_wait();
  int n = 0;
#pragma unroll
  for (int i = 0; i < RUN; i += 256) {
    const int t = blockIdx.x * RUN + i + threadIdx.x;
    if (t < A.T) n += counts(A, t);
  }
  n = __reduce_add_sync(0xffffffffu, n);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x / 32] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    n = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) n += red[i];
    A.runs[blockIdx.x] = n;
  }
}

// The rows that count, side by side in their order; loss and dh of the others are 0.  Each CTA
// counts the rows before its own and all of them by itself, so that one launch does, or takes
// whole runs of them from k_head_runs.
__global__ void __launch_bounds__(256) k_head_rows(const __grid_constant__ Head A) {
  __shared__ int red[2][8];
  __shared__ int live[ROWS];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t0 = blockIdx.x * ROWS, t = t0 + warp;
  const int pieces = A.H / 8, label = t < A.T ? A.labels[t] : -1;
  const float weight = t < A.T ? (A.row_weight ? A.row_weight[t] : 1.f) : 0.f;
  const bool mine = label >= 0 && label < A.V && weight != 0.f;
  int before = 0, all = 0;
  if (A.T <= RUN) {
#pragma unroll 4
    for (int i = threadIdx.x; i < A.T; i += 256) {
      const int c = counts(A, i);
      all += c;
      before += i < t0 ? c : 0;
    }
  } else {
    const int run = t0 / RUN, runs = (A.T + RUN - 1) / RUN;
    for (int i = threadIdx.x; i < runs; i += 256) {
      const int c = A.runs[i];
      all += c;
      before += i < run ? c : 0;
    }
#pragma unroll 4
    for (int i = run * RUN + threadIdx.x; i < min(t0, A.T); i += 256) before += counts(A, i);
  }
  before = __reduce_add_sync(0xffffffffu, before);
  all = __reduce_add_sync(0xffffffffu, all);
  if (lane == 0) red[0][warp] = before, red[1][warp] = all, live[warp] = mine;
  __syncthreads();
  before = all = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    before += red[0][i] + (i < warp ? live[i] : 0);
    all += red[1][i];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *A.n = all;
  if (mine) {
    const uint4* s = (const uint4*)(A.h + (long)t * A.ldh);
    uint4* d = (uint4*)(A.hc + (long)before * A.H);
#pragma unroll 8
    for (int c = lane; c < pieces; c += 32) {
      const uint4 x = s[c];
      d[c] = x;
      if (A.few) ((uint4*)(A.hc + (long)(FEW + before) * A.H))[c] = x;
      if (A.hw && A.hw != A.hc) {
        const float2 f = both(weight);
        ((uint4*)(A.hw + (long)before * A.H))[c] =
            make_uint4(to_bf2(muls(bf2(x.x), f)), to_bf2(muls(bf2(x.y), f)), to_bf2(muls(bf2(x.z), f)), to_bf2(muls(bf2(x.w), f)));
      }
    }
    if (lane == 0) {
      A.label[before] = label;
      A.weight[before] = weight;
      A.row[before] = t;
    }
  } else if (t < A.T) {
    if (lane == 0) A.loss[t] = 0.f;
    if (A.dh) {
      uint4* d = (uint4*)(A.dh + (long)t * A.H);
      for (int c = lane; c < pieces; c += 32) d[c] = make_uint4(0u, 0u, 0u, 0u);
    }
  }
  // rows of the last, ragged block of a sum over the tokens
  if (A.hw && (A.few ? t < 64 && (t >= 2 * FEW || t % FEW >= all) : t >= all && t < (all + 63) / 64 * 64)) {
    uint4* d = (uint4*)(A.hw + (long)t * A.H);
    for (int c = lane; c < pieces; c += 32) d[c] = make_uint4(0u, 0u, 0u, 0u);
  }
}

// A row's log-sum-exp (in units of log 2, as the exponentials are taken) and loss.  A lane a row,
// 32 warps a CTA side by side over the partial sums, added in the warps' order.
__global__ void __launch_bounds__(1024) k_head_lse(const __grid_constant__ Head A) {
  __shared__ float2 red[32][33];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane, n = *A.n;
  if (blockIdx.x * 32 >= n) return;
  // the sums of eight more parts, all taken to the largest value first
  auto join = [](float2& v, const float2 (&p)[8]) {
    float m = v.x;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, p[j].x);
    const float at = m == -INFINITY ? 0.f : m;
    float s = v.y * ex2((v.x - at) * LOG2E);
#pragma unroll
    for (int j = 0; j < 8; ++j) s += p[j].y * ex2((p[j].x - at) * LOG2E);
    v = make_float2(m, s);
  };
  const float2 none = make_float2(-INFINITY, 0.f);
  float2 v = none;
  if (i < n)
    for (int s = warp; s < A.slots; s += 32 * 8) {
      float2 p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = s + 32 * j < A.slots ? A.part[(long)(s + 32 * j) * A.Tp + i] : none;
      join(v, p);
    }
  red[warp][lane] = v;
  __syncthreads();
  if (warp == 0 && i < n) {
    v = none;
#pragma unroll
    for (int w = 0; w < 32; w += 8) {
      float2 p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = red[w + j][lane];
      join(v, p);
    }
    const float l = log2f(v.y), loss = (v.x - A.own[i]) + l * 0.69314718055994531f;
    A.lse2[i] = v.x * LOG2E + l;
    A.loss[A.row[i]] = A.weight[i] * loss;
    A.own[i] = expm1f(-loss);
  }
}

// A block of 32 x 32, a row a lane, into rows of memory (16-byte pieces; those inside the columns
// and for which row() gives a place)
template <typename Row>
__device__ __forceinline__ void put_block(char* stg, const float (&v)[32], __nv_bfloat16* out, long ld, int col0, int cols,
                                          Row row) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *(uint4*)(stg + lane * STG_LD + 16 * j) =
        make_uint4(to_bf2(make_float2(v[8 * j], v[8 * j + 1])), to_bf2(make_float2(v[8 * j + 2], v[8 * j + 3])),
                   to_bf2(make_float2(v[8 * j + 4], v[8 * j + 5])), to_bf2(make_float2(v[8 * j + 6], v[8 * j + 7])));
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = 8 * j + lane / 4, c = col0 + 8 * (lane % 4);
    const long at = row(r);
    if (at >= 0 && c < cols) *(uint4*)(out + at * ld + c) = *(const uint4*)(stg + r * STG_LD + 16 * (lane % 4));
  }
}

// dz of kept logits, a block a warp; rows up to the next 64 are zeros (a sum over the tokens
// takes whole blocks).  Of few tokens, w dz: its values, and FEW rows on what they leave.
__global__ void __launch_bounds__(256) k_head_dz(const __grid_constant__ Head A) {
  __shared__ __align__(16) char stage[8][32 * STG_LD];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = *A.n;
  const int rb = blockIdx.y, cb = blockIdx.x * 8 + warp, at = A.few ? lane % FEW : lane, row = rb * 32 + at;
  if (rb * 32 >= (n + 63) / 64 * 64 || cb >= A.keep_cols) return;
  const float* b = A.keep + ((long)rb * A.keep_cols + cb) * 1024 + at;
  float v[32];
  if (rb * 32 < n) {
#pragma unroll
    for (int e = 0; e < 32; ++e) v[e] = b[32 * e];
  }
  const bool on = row < n;
  const float lse2 = on ? A.lse2[row] : 0.f, own = on ? A.own[row] : 0.f, weight = on && A.few ? A.weight[row] : 1.f;
  const int label = on ? A.label[row] - 32 * cb : -1;
#pragma unroll
  for (int e = 0; e < 32; ++e)
    v[e] = !on ? 0.f : weight * (label == e ? own : ex2(fmaf(v[e], LOG2E, -lse2)));
  if (at != lane) {
#pragma unroll
    for (int e = 0; e < 32; ++e) v[e] -= to_f32(__float2bfloat16_rn(v[e]));
  }
  put_block(stage[warp], v, A.dl, A.ldd, 32 * cb, 32 * A.keep_cols, [&](int r) { return (long)rb * 32 + r; });
}

size_t al(size_t v) { return (v + 255) / 256 * 256; }

// What a call's sizes come to, and where its arrays lie in the workspace
struct Plan {
  long Tp, piece;  // columns of a piece, a multiple of 256
  long Td;         // rows of dz
  int slots, slices;
  size_t hc, hw, label, weight, row, lse2, own, n, runs, part, dl, blocks, keep, bytes;
  int keep_cols;   // blocks of kept logits side by side, 0: not kept
};

Plan plan_of(int T, int V, int H, bool dh, bool dw) {  // (the same with weights and without)
  Plan p = {};
  p.Tp = ((long)T + 255) / 256 * 256;
  const long nt = ((long)V + BN - 1) / BN;
  p.slots = (V + BN / 2 - 1) / (BN / 2);  // halves of tiles that have a column
  p.piece = std::min(nt * BN, std::max(1L, PIECE_BYTES / (2 * p.Tp * BN)) * BN);
  // few tiles of dh: ranges of the vocabulary side by side, so that every pair of SMs has one
  const long tiles = p.Tp / BM * (((long)H + BN - 1) / BN);
  p.slices = (int)std::max(1L, std::min((long)MAX_SLICES, (long)(SMS / 2) / tiles));
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t v = at;
    at += al(n);
    return v;
  };
  p.hc = take(2 * (size_t)p.Tp * H);
  if (dw) p.hw = take(2 * (size_t)p.Tp * H);
  p.label = take(4 * p.Tp);
  p.weight = take(4 * p.Tp);
  p.row = take(4 * p.Tp);
  p.lse2 = take(4 * p.Tp);
  p.own = take(4 * p.Tp);
  p.n = take(4);
  p.runs = take(4 * (p.Tp / RUN + 1));
  p.part = take(8 * (size_t)p.slots * p.Tp);
  p.Td = p.Tp;
  if (dh || dw) {
    const long Tk = ((long)T + 31) / 32 * 32;  // blocks of 32 rows are kept, and dz of 64: no whole tiles
    if (4 * Tk * nt * BN <= PIECE_BYTES) {
      p.keep_cols = (int)(nt * BN / 32);
      p.keep = take(4 * (size_t)Tk * nt * BN);
      p.piece = nt * BN;
      p.Td = ((long)T + 63) / 64 * 64;
    }
    p.dl = take(2 * (size_t)p.Td * p.piece);
  }
  if (dh) p.blocks = take(4 * block_floats(p.Tp, H, p.slices));
  p.bytes = at;
  return p;
}

lx_status check_sizes(int32_t T, int32_t V, int32_t H) {
  if (T < 0) return fail(LX_ERR_ARG, "T < 0");
  if (T > MAX_T) return fail(LX_ERR_SHAPE, "T is above 2^24");
  if (V < 1 || V > MAX_V) return fail(LX_ERR_SHAPE, "V must be in 1..2^24");
  if (H < 8 || H > MAX_H || H % 8 != 0) return fail(LX_ERR_SHAPE, "H must be a multiple of 8 up to 2^20");
  const long tt = ((long)T + 255) / 256, vt = ((long)V + 255) / 256, ht = ((long)H + 255) / 256;
  if (std::max(tt * vt, std::max(tt * ht * 16, vt * ht)) > (1L << 30)) return fail(LX_ERR_SHAPE, "too many tiles");
  return LX_OK;
}

}  // namespace
}  // namespace lx

extern "C" lx_status lx_head_loss_workspace(int32_t T, int32_t V, int32_t H, int32_t want_dh, int32_t want_dw,
                                            uint64_t* bytes) {
  using namespace lx;
  if (!bytes) return fail(LX_ERR_ARG, "bytes is NULL");
  LX_TRY(check_sizes(T, V, H));
  *bytes = T == 0 ? 0 : plan_of(T, V, H, want_dh != 0, want_dw != 0).bytes;
  return LX_OK;
}

extern "C" lx_status lx_head_loss(const void* h, int64_t ldh, const void* w, int64_t ldw, const int32_t* labels,
                                  const float* row_weight, int32_t T, int32_t V, int32_t H, float* loss, void* dh,
                                  void* dw, void* workspace, uint64_t workspace_bytes, void* stream) {
  using namespace lx;
  LX_TRY(check_sizes(T, V, H));
  if (ldh < H || ldh % 8 != 0 || ldh > (1L << 30)) return fail(LX_ERR_SHAPE, "ldh");
  if (ldw < H || ldw % 8 != 0 || ldw > (1L << 30)) return fail(LX_ERR_SHAPE, "ldw");
  if (!w || !aligned(w, 16) || !aligned(h, 16) || !aligned(dh, 16) || !aligned(dw, 16))
    return fail(LX_ERR_ARG, "w is NULL, or h, w, dh or dw not 16-byte aligned");
  if (!aligned(labels, 4) || !aligned(row_weight, 4) || !aligned(loss, 4))
    return fail(LX_ERR_ARG, "a pointer is not aligned to its element");
  cudaStream_t st = (cudaStream_t)stream;
  if (T == 0) {
    if (dw) LX_CUDA(cudaMemsetAsync(dw, 0, 2 * (size_t)V * H, st));
    return LX_OK;
  }
  if (!h || !labels || !loss) return fail(LX_ERR_ARG, "h, labels or loss is NULL");
  const Plan L = plan_of(T, V, H, dh != nullptr, dw != nullptr);
  if (!workspace || !aligned(workspace, 256)) return fail(LX_ERR_ARG, "workspace is NULL or not 256-byte aligned");
  if (workspace_bytes < L.bytes) return fail(LX_ERR_ARG, "workspace too small");
  const void* ins[] = {h, w, labels, row_weight};
  const size_t in_n[] = {span(T, H, ldh, 2), span(V, H, ldw, 2), 4 * (size_t)T, 4 * (size_t)T};
  const void* outs[] = {loss, dh, dw, workspace};
  const size_t out_n[] = {4 * (size_t)T, 2 * (size_t)T * H, 2 * (size_t)V * H, L.bytes};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 4; ++j)
      if (overlap(outs[i], out_n[i], ins[j], in_n[j])) return fail(LX_ERR_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], out_n[i], outs[j], out_n[j])) return fail(LX_ERR_ARG, "two outputs overlap");
  }
  const CallWaits waits = take_call_waits();
  char* ws = (char*)workspace;
  Head A = {};
  A.T = T, A.V = V, A.H = H, A.Tp = (int)L.Tp;
  A.h = (const __nv_bfloat16*)h;
  A.ldh = ldh;
  A.labels = labels;
  A.row_weight = row_weight;
  A.loss = loss;
  A.dh = (__nv_bfloat16*)dh;
  A.hc = (__nv_bfloat16*)(ws + L.hc);
  A.few = L.keep_cols && T <= FEW;
  A.hw = !dw ? nullptr : row_weight && !A.few ? (__nv_bfloat16*)(ws + L.hw) : A.hc;
  A.label = (int*)(ws + L.label);
  A.row = (int*)(ws + L.row);
  A.n = (int*)(ws + L.n);
  A.runs = (int*)(ws + L.runs);
  A.weight = (float*)(ws + L.weight);
  A.lse2 = (float*)(ws + L.lse2);
  A.own = (float*)(ws + L.own);
  A.part = (const float2*)(ws + L.part);
  A.slots = L.slots;
  A.keep = (const float*)(ws + L.keep);
  A.keep_cols = L.keep_cols;
  A.dl = (__nv_bfloat16*)(ws + L.dl);
  A.ldd = L.piece;

  if (T > RUN) LX_TRY(launch_after(k_head_runs, dim3((T + RUN - 1) / RUN), dim3(256), 0, 1, st, A));
  LX_TRY(launch_after(k_head_rows, dim3((unsigned)(L.Tp / ROWS)), dim3(256), 0, 1, st, A));

  Launch P = {};
  P.wait_cycles = waits.cycles;
  P.unmet = waits.unmet == LX_WAIT_CALL_PRODUCT;
  P.n = 1;
  P.label = A.label;
  P.lse2 = A.lse2;
  P.own = A.own;
  P.part = (float2*)(ws + L.part);
  P.part_ld = L.Tp;
  P.keep = L.keep_cols ? (float*)(ws + L.keep) : nullptr;
  P.keep_cols = L.keep_cols;
  Problem& p = P.p[0];
  p.M = (int)L.Tp, p.N = V, p.K = H, p.slices = 1;
  p.rows = A.n;
  if (!operand(&p.a, A.hc, H, L.Tp, H, 2, false) || !operand(&p.b, w, H, V, ldw, 2, false))
    return fail(LX_ERR_CUDA, "cuTensorMapEncodeTiled(head) failed");
  LX_TRY((launch_product<STATS, false>(P, st)));
  LX_TRY(launch_after(k_head_lse, dim3((unsigned)(L.Tp / 32)), dim3(1024), 0, 1, st, A));
  if (!dh && !dw) return LX_OK;

  Launch G = {};
  G.wait_cycles = waits.cycles;
  for (long v0 = 0; v0 < V; v0 += L.piece) {
    const long n = std::min<long>(L.piece, V - v0);
    const __nv_bfloat16* wp = (const __nv_bfloat16*)w + v0 * ldw;
    if (L.keep_cols) {  // (one piece)
      LX_TRY(launch_after(k_head_dz, dim3((L.keep_cols + 7) / 8, (unsigned)(L.Td / 32)), dim3(256), 0, 1, st, A));
    } else {
      P.v0 = (int)v0;
      p.N = (int)((n + 31) / 32 * 32);  // (whole blocks of dz; those behind the vocabulary are not read)
      if (!operand(&p.b, wp, H, n, ldw, 2, false) || !boxes(&P.map_dl, A.dl, L.piece, L.Tp, L.piece)) return fail(LX_ERR_CUDA, "cuTensorMapEncodeTiled(head) failed");
      LX_TRY((launch_product<DLOGIT, false>(P, st)));
    }
    // the gradient with the longer sums first
    G.n = 0;
    bool ok = true;
    for (int i = 0; i < 2; ++i) {
      const bool of_h = (n >= T) == (i == 0);
      if (!(of_h ? dh : dw)) continue;
      Problem& g = G.p[G.n++];
      g = Problem{};
      g.b_mn = 1;
      if (of_h) {
        g.M = A.few ? 2 * FEW : (int)L.Tp, g.N = H, g.K = (int)n, g.slices = L.slices;
        g.rows = A.few ? nullptr : A.n;
        g.blocks = (float*)(ws + L.blocks);
        g.add = v0 > 0;
        ok = ok && operand(&g.a, A.dl, n, L.Td, L.piece, 2, false) && operand(&g.b, wp, H, n, ldw, 2, true);
      } else {
        g.M = (int)n, g.N = H, g.K = (int)L.Tp, g.slices = 1;
        g.a_mn = 1;
        g.depth = A.n;
        ok = ok && boxes(&g.out, (__nv_bfloat16*)dw + v0 * H, H, n, H) &&
             operand(&g.a, A.dl, n, L.Td, L.piece, 2, true) && operand(&g.b, A.hw, H, L.Tp, H, 2, true);
      }
    }
    if (!ok) return fail(LX_ERR_CUDA, "cuTensorMapEncodeTiled(head) failed");
    LX_TRY((launch_product<GRAD, false>(G, st)));
  }
  if (dh) {
    const Join J = {(const float*)(ws + L.blocks), (int)L.Tp, H, L.slices, A.n, A.row, A.few ? nullptr : A.weight, A.dh,
                    A.few ? FEW : 0};
    LX_TRY(launch_join(J, st));
  }
  return LX_OK;
}
