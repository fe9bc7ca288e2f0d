// Helpers of the row-wise operators (block norms, router balance loss,
// distillation): 16-byte or single-element pieces of a row held as fp32, operations on
// pairs of them, sums over a warp, and the entry points' checks of addresses.
#pragma once

#include "lx_internal.cuh"

namespace lx {
namespace rows {

constexpr int SMS = 152;  // of the GPU: shapes grids alone

// VEC fp32 values to consecutive elements at p; VEC * sizeof(T) is 16 (p 16-byte aligned)
// or VEC is 1
template <typename T, int VEC>
__device__ __forceinline__ void store(T* p, const float* v) {
  if constexpr (VEC == 1) {
    *p = from_f32<T>(v[0]);
  } else {
    static_assert(VEC * sizeof(T) == 16, "one 16-byte piece");
    uint32_t w[4];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&b);
      }
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A pair's operations in one instruction (add2, mul2, fma2), each rounded as the single one,
// or in two (adds, muls, fmas).  One instruction takes the issue slot of one but the pipe
// and the latency of two: it won where issue slots bound a kernel (block norms backward: 83
// against 91 us), two where chains of operations did (distillation: 494 and 410 us).
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
      "add.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
      "mul.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 ra, rb, rc, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
      "mov.b64 rc, {%6, %7};\n\tfma.rn.f32x2 rd, ra, rb, rc;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 adds(float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); }
__device__ __forceinline__ float2 muls(float2 a, float2 b) { return make_float2(a.x * b.x, a.y * b.y); }
__device__ __forceinline__ float2 fmas(float2 a, float2 b, float2 c) {
  return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y));
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 bf2(uint32_t w) {  // two bf16: each is the upper half of its fp32
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint32_t to_bf2(float2 v) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(v.x, v.y);
  return *reinterpret_cast<const uint32_t*>(&b);
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Rows `ldb` bytes apart that are copied as the 16-byte blocks they touch: so many rows at either end
// of their array lie so close to it that a block of theirs may reach beyond (a block starts
// up to 15 bytes before its row and ends up to 15 behind it).  ldb = 0: a single row.
__host__ __device__ constexpr uint32_t end_rows(uint32_t ldb) { return ldb == 0 || ldb >= 15 ? 1 : (14 + ldb) / ldb; }

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
// whether [a, a + na) and [b, b + nb) share a byte
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && na && nb && x < y + nb && y < x + na;
}
// bytes from the first to the last element of `T` rows of `n`, `ld` elements apart
inline size_t span(int64_t T, int64_t n, int64_t ld, size_t es) {
  return T > 0 ? ((size_t)(T - 1) * (size_t)ld + (size_t)n) * es : 0;
}

}  // namespace rows
}  // namespace lx
