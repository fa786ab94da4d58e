// mv_row.cuh -- what the kernels over rows of logits share: vectors of elements, packed arithmetic, exponentials and sums.
//
// With z = c x, r a reference near the row's largest logit and t = (x - r) c log2(e):  s = sum 2^t,  lse = c r + log s,
// H = log s - ln 2 (sum 2^t t) / s.  A masked logit (-inf) has 2^t = 0 and must not multiply its t, so t is kept above a
// finite floor.  t is one fused multiply-add, x (c log2 e) - R with R = r c log2(e) rounded; what the rounding of R costs, d = r c
// log2(e) - R, is put right once per thread by 2^-d to the second order, and so only while |R| stays below R_MAX: there |d| <= 2^-7
// and (d ln 2)^3 / 6 < 2.7e-8, half a unit of 32 bits.  Parts whose logits times c log2(e) all lie below -R_MAX, or some above
// R_MAX (a whole row masked by a finite fill, an inverse temperature of 1e5), are summed again in a form that takes the difference first.

#pragma once
#include "mv_lm.cuh"

#include <cooperative_groups.h>
#include <math.h>
#include <string.h>
#include <type_traits>

namespace {

namespace cg = cooperative_groups;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float T_FLOOR = -1.0e4f;    // 2^t is 0 far above it, and a sum of 2^31 terms of up to 2^10 times it is finite
constexpr float R_MAX = 131072.0f;   // references of at most this magnitude are summed by the fused form
constexpr float C2_MIN = 1.0e-30f;   // below that scale the distances that count are not small beside the type's range
constexpr float LAG = 10.0f;         // a logit changes a thread's reference only if it exceeds it by 2^LAG

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Two 32-bit numbers in one register pair: one instruction for both.
typedef unsigned long long f2;
__device__ __forceinline__ f2 pack2(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(f2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// 16 bytes of logits: the larger halves of two words (a NaN is never the larger), the larger half of one, and the elements two by two.
template <typename X> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static constexpr uint32_t NONE = 0xff800000u;                       // -inf
  __device__ static uint32_t max2(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
  __device__ static float widen(uint32_t m) { return __uint_as_float(m); }
  __device__ static f2 pair(const uint4& u, int i) {
    return i == 0 ? pack2(__uint_as_float(u.x), __uint_as_float(u.y)) : pack2(__uint_as_float(u.z), __uint_as_float(u.w));
  }
};
__device__ __forceinline__ uint32_t word(const uint4& u, int i) { return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w; }
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static constexpr uint32_t NONE = 0xff80ff80u;
  __device__ static uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  __device__ static uint32_t max2_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  __device__ static float widen(uint32_t m) { return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u)); }
  __device__ static f2 pair(const uint4& u, int i) {
    const uint32_t w = word(u, i);
    return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
};
template <> struct Vec<__half> {
  static constexpr int N = 8;
  static constexpr uint32_t NONE = 0xfc00fc00u;
  __device__ static uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  __device__ static float2 both(uint32_t w) {
    __half2 h;
    memcpy(&h, &w, 4);
    return __half22float2(h);
  }
  __device__ static float widen(uint32_t m) {
    const float2 f = both(m);
    return fmaxf(f.x, f.y);
  }
  __device__ static f2 pair(const uint4& u, int i) {
    const float2 f = both(word(u, i));
    return pack2(f.x, f.y);
  }
};

// 16 bytes that begin `shift` bytes (even, below 16) into two neighbouring vectors.
__device__ __forceinline__ uint4 between(const uint4& lo, const uint4& hi, int shift) {
  const bool two = shift & 8, one = shift & 4;
  const int bits = shift % 4 * 8;
  const uint32_t a0 = two ? lo.z : lo.x, a1 = two ? lo.w : lo.y, a2 = two ? hi.x : lo.z, a3 = two ? hi.y : lo.w, a4 = two ? hi.z : hi.x, a5 = two ? hi.w : hi.y;
  const uint32_t b0 = one ? a1 : a0, b1 = one ? a2 : a1, b2 = one ? a3 : a2, b3 = one ? a4 : a3, b4 = one ? a5 : a4;
  return make_uint4(__funnelshift_r(b0, b1, bits), __funnelshift_r(b1, b2, bits), __funnelshift_r(b2, b3, bits), __funnelshift_r(b3, b4, bits));
}

// 32 bytes at a multiple of 32: a whole sector.
__device__ __forceinline__ void load_stream(const uint4* p, uint4& a, uint4& b) {
  asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(p));
}

template <typename X, typename F> __device__ __forceinline__ void each_logit(const uint4& u, F&& f) {
#pragma unroll
  for (int i = 0; i < Vec<X>::N / 2; ++i) {
    float a, b;
    unpack2(Vec<X>::pair(u, i), a, b);
    f(2 * i, a);
    f(2 * i + 1, b);
  }
}

// ------------------------------------------------------------------------------------------ narrowing
template <typename X> __device__ __forceinline__ uint32_t narrow2(float a, float b);
template <> __device__ __forceinline__ uint32_t narrow2<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  uint32_t r;
  memcpy(&r, &h, 4);
  return r;
}
template <> __device__ __forceinline__ uint32_t narrow2<__half>(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  uint32_t r;
  memcpy(&r, &h, 4);
  return r;
}

template <typename X> __device__ __forceinline__ uint4 pack_vec(const float (&d)[Vec<X>::N]) {
  if constexpr (sizeof(X) == 4) return make_uint4(__float_as_uint(d[0]), __float_as_uint(d[1]), __float_as_uint(d[2]), __float_as_uint(d[3]));
  else return make_uint4(narrow2<X>(d[0], d[1]), narrow2<X>(d[2], d[3]), narrow2<X>(d[4], d[5]), narrow2<X>(d[6], d[7]));
}

// ------------------------------------------------------------------------------------------ rows
// (value descending, index ascending) as one number, larger is earlier; +0 and -0 are one value.  0 is no key.
__device__ __forceinline__ unsigned long long make_key(float x, uint32_t idx) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return (unsigned long long)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (0xffffffffu - idx);
}
__device__ __forceinline__ float key_value(unsigned long long k) {
  const uint32_t h = uint32_t(k >> 32);
  return __uint_as_float(h & 0x80000000u ? h & 0x7fffffffu : ~h);
}
__device__ __forceinline__ uint32_t key_index(unsigned long long k) { return 0xffffffffu - uint32_t(k); }

// One row, or one CTA's part of it: `head` single logits, nv vectors of 16 bytes (an even number, from a multiple of 32 bytes
// on), `tail` single logits.
template <typename X> struct Part {
  const X* row;
  const uint4* vec;                  // the part's first vector
  int64_t nv;
  uint32_t col0;                     // its column
  uint32_t head, tail, tail_col;
};

struct Sums { float ref, s, st; };   // s = sum 2^t, st = sum 2^t t, both relative to ref (-inf: nothing yet)

// (a - b) c of two logits; a quarter of each where the difference could pass the range of 32 bits and count all the same
__device__ __forceinline__ float distance(float a, float b, float c) {
  return c < 1.0f ? (0.25f * a - 0.25f * b) * (4.0f * c) : (a - b) * c;
}

// The same sums relative to a larger reference.
__device__ __forceinline__ Sums shift(const Sums& x, float ref, float c2) {
  const float d = ref == x.ref ? 0.0f : max_nan(distance(x.ref, ref, c2), T_FLOOR);
  const float f = exp2_fast(d);
  return {ref, x.s * f, fmaf(x.s, d, x.st) * f};
}

// The sums of a part whose reference does not fit the fused form (or that is empty), by differences to its largest logit m (every
// thread has the largest of its own): one more reading of the part.
template <typename X, int TPB>
__device__ __noinline__ Sums sums_of_extremes(const Part<X>& p, float c2, float m, float* sh) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  __syncthreads();
  if (lane == 0) sh[w] = m;
  __syncthreads();
  for (int i = 0; i < TPB / 32; ++i) m = fmaxf(m, sh[i]);
  const float ref = m == -INFINITY ? 0.0f : m;
  Sums x = {m, 0.0f, 0.0f};
  auto add = [&](float v) {
    const float u = max_nan(distance(v, ref, c2), T_FLOOR), e = exp2_fast(u);
    x.s += e;
    x.st = fmaf(e, u, x.st);
  };
  if (threadIdx.x < p.head + p.tail) add(to_f(p.row[threadIdx.x < p.head ? threadIdx.x : p.tail_col + threadIdx.x - p.head]));
  for (int64_t v = threadIdx.x; v < p.nv; v += TPB) each_logit<X>(__ldg(p.vec + v), [&](int, float x) { add(x); });
  __syncthreads();
  return x;
}

}  // namespace
