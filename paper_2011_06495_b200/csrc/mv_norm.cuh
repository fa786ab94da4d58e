// mv_norm.cuh -- what layer norm and its gradients share: units of a row, sums over lanes, parameters, shapes of CTAs.
#pragma once
#include "mv_row.cuh"

namespace {

// A row is read once, into registers, by L lanes (of a part of a warp, or of several), each with up to NV units: vectors of 16 bytes where
// rows lie on their boundaries, single elements elsewhere (in the gradient, whose columns belong to threads).  Arithmetic is on two
// elements at a time: 20 instructions an element in the gradient instead of 32 (65536 x 2048 bf16, in short runs: 140 us instead of 181).
template <typename X, bool VEC> struct Unit;
template <typename X> struct Unit<X, true> {
  static constexpr int N = Vec<X>::N;
  uint4 u;
  __device__ __forceinline__ void load(const X* p) { u = __ldcs(reinterpret_cast<const uint4*>(p)); }
};
template <typename X> struct Unit<X, false> {
  static constexpr int N = 1;
  X u;
};

// The pairs of a thread's units, of which `n` hold something: f(unit, pair in it, pair's number, whether the second element counts).
template <typename X, bool VEC, int NV, typename F> __device__ __forceinline__ void each_pair(int n, F&& f) {
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (i >= n) break;
#pragma unroll
      for (int j = 0; j < Vec<X>::N / 2; ++j) f(i, j, i * (Vec<X>::N / 2) + j, true);
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV / 2; ++j) {
      if (2 * j >= n) break;
      f(2 * j, 0, j, 2 * j + 1 < n);
    }
  }
}

// Writes f of every pair, its arguments as above, to a row from p on.
template <typename X, bool VEC, int NV, int L, typename F> __device__ __forceinline__ void put_pairs(int n, X* p, F&& f) {
  if constexpr (VEC) {
    constexpr int N = Vec<X>::N;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (i >= n) break;
      float o[N];
#pragma unroll
      for (int j = 0; j < N / 2; ++j) unpack2(f(i, j, i * (N / 2) + j, true), o[2 * j], o[2 * j + 1]);
      __stcs(reinterpret_cast<uint4*>(p + i * L * N), pack_vec<X>(o));
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV / 2; ++j) {
      if (2 * j >= n) break;
      const bool second = 2 * j + 1 < n;
      float a, b;
      unpack2(f(2 * j, 0, j, second), a, b);
      p[2 * j * L] = from_f<X>(a);
      if (second) p[(2 * j + 1) * L] = from_f<X>(b);
    }
  }
}
// The pair j of a vector, or the pair that begins with element i.
template <typename X, bool VEC, typename G> __device__ __forceinline__ f2 pair_of(G&& get, int i, int j, bool second) {
  if constexpr (VEC) return Vec<X>::pair(get(i).u, j);
  else return pack2(to_f(get(i).u), second ? to_f(get(i + 1).u) : 0.0f);
}
__device__ __forceinline__ float add_up(f2 v) {
  float a, b;
  unpack2(v, a, b);
  return a + b;
}
__device__ __forceinline__ f2 both(float v) { return pack2(v, v); }

// The sum over L neighbouring lanes, for each of them.
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = L / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

__device__ __forceinline__ float parameter(const void* p, int type, int64_t i, float none) {
  if (!p) return none;
  return type == MV_F32 ? static_cast<const float*>(p)[i] : type == MV_BF16 ? to_f(static_cast<const __nv_bfloat16*>(p)[i]) : to_f(static_cast<const __half*>(p)[i]);
}

// A sum over D, times a rounded 1 / D, leaves the mean m off by e, which beside a small spread is not little (1000 columns of 1000.0: 6e-5; y 0.02
// instead of 0).  The pass over d = x - m adds up d beside d^2: e = mean d, v = mean d^2 - e^2, and y's (d - e) r is d r + shift.
struct Centre { float mean, rstd, shift; };
__device__ __forceinline__ Centre centre(float m, float sum_d, float sum_d2, float share, float eps) {
  const float e = fabsf(sum_d) < INFINITY ? sum_d * share : 0.0f, r = rsqrtf(max_nan(fmaf(-e, e, sum_d2 * share), 0.0f) + eps);
  return {m + e, r, -e * r};
}

// Parameters in shared memory, unit by unit; of units of eight the first fours, then the second fours, so that neighbouring lanes read
// neighbouring 16 bytes.
template <int N> __device__ __forceinline__ int place(int i, int units) { return N == 8 ? (((i >> 2) & 1) * units + (i >> 3)) * 4 + (i & 3) : i; }
// The parameters of pair k (as in each_pair) of the lane `at`.
template <int N, int L> __device__ __forceinline__ f2 param_pair(const float* p, int at, int units, int k, bool second) {
  if constexpr (N == 1) {
    const float* q = p + at + 2 * k * L;
    return pack2(q[0], second ? q[L] : 0.0f);
  } else {
    const int i = k / (N / 2), j = k % (N / 2);
    const ulonglong2 q = reinterpret_cast<const ulonglong2*>(p)[(j / 2) * units + at + i * L];
    return j % 2 ? q.y : q.x;
  }
}

// D parameters to their places, eight loads of a thread on their way at once.
template <int N, typename W> __device__ __forceinline__ void put_typed(float* to, const W* from, int D, int units) {
  for (int i0 = threadIdx.x; i0 < D; i0 += 8 * blockDim.x) {
    W v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i0 + j * int(blockDim.x) < D) v[j] = from[i0 + j * blockDim.x];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i0 + j * int(blockDim.x) < D) to[place<N>(i0 + j * blockDim.x, units)] = to_f(v[j]);
  }
}
template <int N> __device__ __forceinline__ void put_params(float* to, const void* p, int type, float none, int D, int units) {
  if (!p)
    for (int i = threadIdx.x; i < D; i += blockDim.x) to[i] = none;
  else if (type == MV_F32) put_typed<N>(to, static_cast<const float*>(p), D, units);
  else if (type == MV_BF16) put_typed<N>(to, static_cast<const __nv_bfloat16*>(p), D, units);
  else put_typed<N>(to, static_cast<const __half*>(p), D, units);
}

constexpr int NORM_TPB = 256, WIDE_TPB = 512;

// Waits for the L threads of one group.
template <int L> __device__ __forceinline__ void group_sync(int group) {
  if constexpr (L > 32) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(L) : "memory");
  else __syncwarp();
}

// Rows of any length: three readings.
constexpr int LONG_TPB = 512;
__device__ __forceinline__ float cta_sum(float v, float* sh) {
  v = lanes_sum<32>(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0f;
  for (int i = 0; i < LONG_TPB / 32; ++i) v += sh[i];
  return v;
}

// How rows of `units` are shared: by few lanes with many units each where there are many rows, by many lanes where there are few.
struct Shape { int lanes, nv; };

constexpr int MANY_ROWS = 148 * 8;

inline int pow2_at_least(int64_t n) {
  int p = 1;
  while (p < n) p *= 2;
  return p;
}

// All of them powers of two; `liked`: units per lane where there are many rows.
inline bool norm_shape(int64_t units, int64_t T, int least_lanes, int most_lanes, int least, int liked, int most, Shape* s) {
  if (units > int64_t(most_lanes) * most) return false;
  const int want = T >= MANY_ROWS ? liked : least;
  int64_t lanes = pow2_at_least((units + want - 1) / want);
  lanes = lanes < least_lanes ? least_lanes : lanes > most_lanes ? most_lanes : lanes;
  s->nv = pow2_at_least((units + lanes - 1) / lanes);
  if (s->nv < least) s->nv = least;
  s->lanes = int(lanes);
  return true;
}

// Calls f with the lanes and units as constants; only the pairs that norm_shape can give.
template <int I> using Int = std::integral_constant<int, I>;
template <int LANES, bool ALL, int NV, int LIKED, int MOST, typename F> int with_units(int nv, F&& f) {
  if constexpr (NV >= MOST) return f(Int<LANES>(), Int<MOST>());
  else return nv <= NV ? f(Int<LANES>(), Int<NV>()) : with_units<LANES, ALL, ALL ? NV * 2 : LIKED, LIKED, MOST>(nv, f);
}
template <int LANES, int MOST_LANES, int LEAST, int LIKED, int MOST, int FEWEST, typename F> int with_shape(const Shape& s, F&& f) {
  if constexpr (LANES < MOST_LANES) {
    if (s.lanes != LANES) return with_shape<LANES * 2, MOST_LANES, LEAST, LIKED, MOST, FEWEST>(s, f);
  }
  return with_units<LANES, LANES == FEWEST || LANES == MOST_LANES, LEAST, LIKED, LANES == MOST_LANES ? MOST : LIKED>(s.nv, f);
}

inline bool unaligned(const void* p, int64_t rows, int64_t ld, int size) { return misaligned(p, 16) || (rows > 1 && ld * size % 16 != 0); }

inline bool bad_rows(const void* p, int type, int64_t ld, int64_t T, int64_t D) { return (T > 0 && !p) || ld < D || misaligned(p, type_size(type)); }

}  // namespace
