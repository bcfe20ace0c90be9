// Rows of bf16, fp16 or fp32 taken eight elements at a time, sums over a CTA, and the rounding of a row to int8: shared by
// the kernels of the 8-bit products and of the norms.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "armor_internal.cuh"

namespace rows {

template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

// two 16-bit values in a register, the first in its low half
__device__ __forceinline__ float2 unpack2(const __nv_bfloat16*, uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack2(const __half*, uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ uint32_t pack2(const __nv_bfloat16*, float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack2(const __half*, float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Two floats as two bf16 numbers each: the nearest one, and what is missing rounded towards zero, 15 bits or more together.  (The rest stays
// below a half step of the first number where it was, so that the sum of the two rounds to bf16 as the float does.)  A first number
// that is not finite stands alone.
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
  const __nv_bfloat16* t = nullptr;
  hi = pack2(t, a, b);
  const float2 h = unpack2(t, hi);
  const float ra = fabsf(h.x) < __int_as_float(0x7f800000) ? a - h.x : 0.f, rb = fabsf(h.y) < __int_as_float(0x7f800000) ? b - h.y : 0.f;
  lo = __byte_perm(__float_as_uint(ra), __float_as_uint(rb), 0x7632);
}

// Eight consecutive elements as they lie: a chunk of a row that waits in registers.
template <typename T> struct Raw8 { uint4 w; };
template <> struct Raw8<float> { float4 a, b; };

template <typename T>
__device__ __forceinline__ Raw8<T> raw_load(const T* p) { return {*reinterpret_cast<const uint4*>(p)}; }
__device__ __forceinline__ Raw8<float> raw_load(const float* p) {
  return {*reinterpret_cast<const float4*>(p), *reinterpret_cast<const float4*>(p + 4)};
}
template <typename T>
__device__ __forceinline__ void raw_get(const Raw8<T>& r, float (&v)[8]) {
  const uint32_t w[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = unpack2(static_cast<const T*>(nullptr), w[i]);
    v[2 * i] = f.x; v[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ void raw_get(const Raw8<float>& r, float (&v)[8]) {
  v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w; v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}
template <typename T>
__device__ __forceinline__ Raw8<T> raw_zero() { return {make_uint4(0u, 0u, 0u, 0u)}; }
template <>
__device__ __forceinline__ Raw8<float> raw_zero<float>() { return {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)}; }

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  const T* t = nullptr;
  *reinterpret_cast<uint4*>(p) = make_uint4(pack2(t, v[0], v[1]), pack2(t, v[2], v[3]), pack2(t, v[4], v[5]), pack2(t, v[6], v[7]));
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// ---------------------------------------------------------------- pairs of floats: one instruction for two
typedef unsigned long long F2;
__device__ __forceinline__ F2 f2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ F2 f2(float a) { return f2(a, a); }
__device__ __forceinline__ float2 f2_get(F2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float f2_sum(F2 v) { const float2 f = f2_get(v); return f.x + f.y; }
// U elements (four or eight) from or to 16-byte (fp32, or eight 16-bit) or 8-byte boundaries.  Rows with fp32 are taken by fours: neighbouring
// lanes then touch neighbouring 16 bytes, where by eights they would meet in the same banks of shared memory and write half sectors.
template <int U, typename T>
__device__ __forceinline__ void get_u(const T* p, F2 (&v)[U / 2]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < U / 4; ++k) {
      const float4 f = *reinterpret_cast<const float4*>(p + 4 * k);
      v[2 * k] = f2(f.x, f.y); v[2 * k + 1] = f2(f.z, f.w);
    }
  } else {
    uint32_t w[U / 2];
    if constexpr (U == 8) {
      const uint4 r = *reinterpret_cast<const uint4*>(p);
      w[0] = r.x; w[1] = r.y; w[2] = r.z; w[3] = r.w;
    } else {
      const uint2 r = *reinterpret_cast<const uint2*>(p);
      w[0] = r.x; w[1] = r.y;
    }
#pragma unroll
    for (int i = 0; i < U / 2; ++i) { const float2 f = unpack2(static_cast<const T*>(nullptr), w[i]); v[i] = f2(f.x, f.y); }
  }
}
template <int U, typename T>
__device__ __forceinline__ void put_u(T* p, const F2 (&v)[U / 2]) {
  float2 f[U / 2];
#pragma unroll
  for (int i = 0; i < U / 2; ++i) f[i] = f2_get(v[i]);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < U / 4; ++k) *reinterpret_cast<float4*>(p + 4 * k) = make_float4(f[2 * k].x, f[2 * k].y, f[2 * k + 1].x, f[2 * k + 1].y);
  } else {
    const T* t = nullptr;
    if constexpr (U == 8) *reinterpret_cast<uint4*>(p) = make_uint4(pack2(t, f[0].x, f[0].y), pack2(t, f[1].x, f[1].y), pack2(t, f[2].x, f[2].y), pack2(t, f[3].x, f[3].y));
    else *reinterpret_cast<uint2*>(p) = make_uint2(pack2(t, f[0].x, f[0].y), pack2(t, f[1].x, f[1].y));
  }
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }

// Elements e .. e + 7 of a row of n, zeros behind its end.  ALIGNED: rows start on 16-byte boundaries, so that only the last chunk of
// a row whose length is no multiple of eight is taken element by element; else all are.
template <bool ALIGNED, typename T>
__device__ __forceinline__ Raw8<T> row_load(const T* row, int64_t e, int64_t n) {
  if (ALIGNED && e + 8 <= n) return raw_load(row + e);
  Raw8<T> r = raw_zero<T>();
  T* const at = reinterpret_cast<T*>(&r);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (e + i < n) at[i] = row[e + i];
  return r;
}
template <bool ALIGNED, typename T>
__device__ __forceinline__ void row_store(T* row, int64_t e, int64_t n, const float (&v)[8]) {
  if (ALIGNED && e + 8 <= n) { store8(row + e, v); return; }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (e + i < n) row[e + i] = from_f<T>(v[i]);
}

// ---------------------------------------------------------------- sums and maxima over a CTA of up to 32 warps
// `buf` holds 32 values per use; a use may follow another on another buffer with no barrier of its own between.
template <int N>
__device__ __forceinline__ void cta_sums(float (&v)[N], float (*buf)[32]) {
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane < N) {
    float mine = v[0];
#pragma unroll
    for (int k = 1; k < N; ++k) if (lane == k) mine = v[k];
    buf[lane][warp] = mine;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    float t = lane < warps ? buf[k][lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    v[k] = t;
  }
}
__device__ __forceinline__ unsigned cta_max(unsigned v, float (*buf)[32]) {
  v = __reduce_max_sync(0xffffffffu, v);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) buf[0][warp] = __uint_as_float(v);
  __syncthreads();
  return __reduce_max_sync(0xffffffffu, lane < warps ? __float_as_uint(buf[0][lane]) : 0u);
}

// ---------------------------------------------------------------- a row as int8 with one scale
// s = a / 127 with a the row's largest |x|, q = the integer next to 127 x / a, ties to even.  x times 127 / a (rounded) is off from that
// quotient by at most 127 x 2^-24 = 7.6e-6, so where it lies further than 2e-5 from a half its nearest integer is right: added to 1.5 x 2^23 in
// one rounding, that integer is the low byte of the sum.  Nearer to a half, 127 x and (k + 1/2) a are compared as 64-bit products, which
// hold them exactly (31 and 33 bits).  q is the exact one for every input, so the order of a sum or another instruction never moves
// it.  (An instruction or two a step for each element, as floor, compare and convert, 60 us where this takes 30: 4,096 x 8,192 in a product's way out.)
struct RowScale {
  float pre;             // a power of two that brings the row into the middle of the exponent range; 0: the row's integers are zeros
  float inv, top;        // 127 / (a pre), a pre
  float s;               // the scale
  float edge;            // distance from an integer beyond which an element is looked at closely; -1: all are (pre is not 1); 2: none is
};
// top_bits: the largest |x| as bits; at least those of infinity: the row holds a NaN or an infinity.  Such a row gets NaN as its
// scale, so that what is made of it is NaN, and zeros; a row of zeros gets 0.
//
// SHORT: a row of bf16 or fp16, whose significands are whole numbers X, A below 2^11.  With s the difference of the exponents, 127 x / a is off from a
// half by |254 X - (2k + 1) A 2^s| / (2 A 2^s), so it is a half or further from it than 1 / (2 A 2^s), which is 16 times the error of x
// times an inverse that is a rounding off (127 X / (A 2^s) x 2^-23).  A half needs 127 to divide (2k + 1) A: unless it divides A, only x = a / 2 is
// one, 63.5 steps, which an inverse rounded up brings to the even 64.  So nothing is looked at closely (of bf16 rows one element in
// a thousand is half of the largest, and the whole warp waits for its comparison: 4,096 x 8,192 bf16 33.0 us, so 25.5).
template <bool SHORT = false>
__device__ __forceinline__ RowScale row_scale(unsigned top_bits) {
  RowScale r;
  const float a = __uint_as_float(top_bits);
  if (top_bits >= 0x7f800000u) return {0.f, 0.f, 1.f, __uint_as_float(0x7fffffffu), -1.f};
  if (top_bits == 0u) return {0.f, 0.f, 1.f, 0.f, -1.f};
  r.pre = a < 1e-18f ? 1.2676506002282294e30f : (a > 1e18f ? 7.8886090522101181e-31f : 1.f);    // 2^100, 2^-100
  r.top = a * r.pre;
  r.inv = __fdiv_rn(127.f, r.top);
  r.s = __fdiv_rn(a, 127.f);
  r.edge = r.pre == 1.f ? 0.49998f : -1.f;
  if (SHORT && r.pre == 1.f && ((top_bits & 0x7fffffu) | 0x800000u) % 127u != 0u) {
    r.inv = __fdiv_ru(127.f, r.top);
    r.edge = 2.f;
  }
  return r;
}
static __device__ __noinline__ int row_round(float x, float pre, float inv, float top) {
  if (pre == 0.f) return 0;
  const float xs = x * pre, t = xs * inv, k = floorf(t);
  if (fabsf(t - k - 0.5f) > 4e-5f) return __float2int_rn(t);
  const double d = 127.0 * (double)xs - ((double)k + 0.5) * (double)top;
  const int f = (int)k;
  return d > 0.0 ? f + 1 : (d < 0.0 ? f : f + (f & 1));
}
__device__ __forceinline__ int row_round(float x, const RowScale& r) { return row_round(x, r.pre, r.inv, r.top); }
// N elements (four or eight), two at a time.  SHORT: row_scale's.
template <int N, bool SHORT>
__device__ __forceinline__ void row_round_n(const float* v, const RowScale& r, uint32_t (&w)[N / 4]) {
  const F2 M = f2(12582912.f), inv = f2(r.inv), minus = f2(-1.f);            // 1.5 x 2^23: its neighbours are whole numbers
  float2 b[N / 2];
  float far = 0.f;
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const F2 x = f2(v[2 * i], v[2 * i + 1]), sum = f2_fma(x, inv, M);
    b[i] = f2_get(sum);
    if (SHORT && r.edge > 1.f) continue;
    const float2 off = f2_get(f2_fma(x, inv, f2_fma(sum, minus, M)));        // (M - sum is exact)
    far = fmaxf(far, fmaxf(fabsf(off.x), fabsf(off.y)));
  }
#pragma unroll
  for (int k = 0; k < N / 4; ++k)
    w[k] = __byte_perm(__byte_perm(__float_as_uint(b[2 * k].x), __float_as_uint(b[2 * k].y), 0x0040),
                       __byte_perm(__float_as_uint(b[2 * k + 1].x), __float_as_uint(b[2 * k + 1].y), 0x0040), 0x5410);
  if (far > r.edge) {
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
      w[k] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[k] |= (uint32_t)(row_round(v[4 * k + i], r) & 255) << (8 * i);
    }
  }
}
__device__ __forceinline__ uint32_t row_round4(const float* v, const RowScale& r) {
  uint32_t w[1];
  row_round_n<4, false>(v, r, w);
  return w[0];
}
template <bool SHORT = false>
__device__ __forceinline__ uint2 row_round8(const float (&v)[8], const RowScale& r) {
  uint32_t w[2];
  row_round_n<8, SHORT>(v, r, w);
  return make_uint2(w[0], w[1]);
}
// the bits of max |v|: of floats without their sign, NaN above infinity above all others
__device__ __forceinline__ unsigned abs_bits8(const float (&v)[8]) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
}

// The same of a chunk as it lies.  16-bit values without their signs stand in the order of their bits, NaN above infinity: two at a time.
template <typename T>
__device__ __forceinline__ unsigned raw_top(const Raw8<T>& r) {
  auto most = [](uint32_t a, uint32_t b) {
    uint32_t m;
    asm("max.u16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
  };
  constexpr uint32_t ABS = 0x7fff7fffu;
  const uint32_t m = most(most(r.w.x & ABS, r.w.y & ABS), most(r.w.z & ABS, r.w.w & ABS));
  const float2 f = unpack2(static_cast<const T*>(nullptr), max(m & 0xffffu, m >> 16));
  return __float_as_uint(f.x);
}
__device__ __forceinline__ unsigned raw_top(const Raw8<float>& r) {
  float v[8];
  raw_get(r, v);
  return abs_bits8(v);
}

inline bool aligned16(const void* p, int64_t ld, int esize) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * esize % 16 == 0; }

}  // namespace rows
