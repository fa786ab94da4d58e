// mv_norm.cu -- layer norm of rows and its gradients, for sm_100a.

#include "mv_row.cuh"

namespace {

// A row is read once, into registers, by L lanes (of a part of a warp, or of several), each with up to NV units: vectors of 16 bytes where
// rows lie on their boundaries, single elements elsewhere.  Arithmetic is on two elements at a time.
template <typename X, bool VEC> struct Unit;
template <typename X> struct Unit<X, true> {
  static constexpr int N = Vec<X>::N;
  uint4 u;
  __device__ __forceinline__ void load(const X* p) { u = __ldcs(reinterpret_cast<const uint4*>(p)); }
};
template <typename X> struct Unit<X, false> {
  static constexpr int N = 1;
  X u;
  __device__ __forceinline__ void load(const X* p) { u = *p; }
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

struct NormArgs {
  int64_t T, D, ldx, ldy;
  const void *weight, *bias;
  int w_type;
  float eps;
  float *mean, *rstd;
  int64_t per;                       // rows per CTA
};

constexpr int NORM_TPB = 256, WIDE_TPB = 512;

// Waits for the L threads of one group.
template <int L> __device__ __forceinline__ void group_sync(int group) {
  if constexpr (L > 32) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(L) : "memory");
  else __syncwarp();
}

// Threads at work at once decide how many bytes are on their way: CTAs per multiprocessor that the registers allow.
constexpr int norm_resident(int elements, bool wide) { return elements > 16 ? (wide ? 1 : 2) : wide ? 2 : elements > 8 ? 4 : 6; }

template <typename X, int L, int NV>
__global__ void __launch_bounds__(L > 32 ? WIDE_TPB : NORM_TPB, norm_resident(NV * Unit<X, true>::N, L > 32)) k_norm(const X* x, X* y, const __grid_constant__ NormArgs a) {
  using Un = Unit<X, true>;
  constexpr int N = Un::N, GROUPS = (L > 32 ? WIDE_TPB : NORM_TPB) / L, WARPS = L / 32;
  extern __shared__ float4 params[];         // weights, then biases
  __shared__ float part[2][WIDE_TPB / 32];
  const int D = int(a.D), units = D / N, mine = threadIdx.x / L, at = threadIdx.x % L;
  const int n = units > at ? (units - at - 1) / L + 1 : 0;
  float* pw = reinterpret_cast<float*>(params);
  float* pb = pw + (D + 3) / 4 * 4;
  const int64_t t0 = blockIdx.x * a.per, t1 = min(a.T, t0 + a.per);
  Un next[NV], u[NV];
  auto load = [&](int64_t t) {
    const X* p = x + t * a.ldx + at * N;
    const int any = t < t1 ? n : 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < any) next[i].load(p + i * L * N);
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) next[i] = Un();
  load(t0 + mine);
  put_params<N>(pw, a.weight, a.w_type, 1.0f, D, units);
  put_params<N>(pb, a.bias, a.w_type, 0.0f, D, units);
  __syncthreads();
  auto sum = [&](float v, int k) {
    v = lanes_sum<(L < 32 ? L : 32)>(v);
    if constexpr (WARPS > 1) {
      if ((threadIdx.x & 31) == 0) part[k][threadIdx.x >> 5] = v;
      group_sync<L>(mine);
      v = 0.0f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) v += part[k][mine * WARPS + i];
    }
    return v;
  };
  auto get = [&](int i) -> const Un& { return u[i]; };
  const float share = 1.0f / float(D);
  for (int64_t r = t0; r < t1; r += GROUPS) {
    const int64_t t = r + mine;
#pragma unroll
    for (int i = 0; i < NV; ++i) u[i] = next[i];
    load(t + GROUPS);
    f2 s = both(0.0f);
    each_pair<X, true, NV>(n, [&](int i, int j, int, bool second) { s = add2(s, pair_of<X, true>(get, i, j, second)); });
    const float mu = sum(add_up(s), 0) * share;
    const f2 minus = both(-mu);
    s = both(0.0f);
    each_pair<X, true, NV>(n, [&](int i, int j, int, bool second) {
      const f2 d = add2(pair_of<X, true>(get, i, j, second), minus);
      s = fma2(d, d, s);
    });
    const float rs = rsqrtf(fmaf(sum(add_up(s), 1), share, a.eps));
    if (t >= t1) continue;
    const f2 rs2 = both(rs);
    put_pairs<X, true, NV, L>(n, y + t * a.ldy + at * N, [&](int i, int j, int k, bool second) {
      return fma2(mul2(add2(pair_of<X, true>(get, i, j, second), minus), rs2), param_pair<N, L>(pw, at, units, k, second), param_pair<N, L>(pb, at, units, k, second));
    });
    if (at == 0) {
      if (a.mean) a.mean[t] = mu;
      if (a.rstd) a.rstd[t] = rs;
    }
  }
}

// Rows that do not lie on 16-byte boundaries.  The vectors are those of y's row, from its first boundary on (in every row another column); what is
// before and behind them, up to 31 elements, goes to a lane each.  APART: x lies otherwise within 16 bytes, and comes from between
// two of its vectors.  Weight and bias of a column side by side, those of every N-th column together, so that neighbouring lanes
// read neighbouring pairs wherever the vectors begin.
template <typename X, bool APART, int L, int NV>
__global__ void __launch_bounds__(L > 32 ? WIDE_TPB : NORM_TPB, L > 32 ? 1 : 2) k_norm_any(const X* x, X* y, const __grid_constant__ NormArgs a) {
  constexpr int N = Vec<X>::N, GROUPS = (L > 32 ? WIDE_TPB : NORM_TPB) / L, WARPS = L / 32, SIZE = sizeof(X), ENDS = L < 32 ? 32 / L : 1;
  extern __shared__ float2 pairs[];
  __shared__ float part[2][WIDE_TPB / 32];
  const int D = int(a.D), columns = (D + N - 1) / N, mine = threadIdx.x / L, at = threadIdx.x % L;
  const int64_t t0 = blockIdx.x * a.per, t1 = min(a.T, t0 + a.per);
  struct Row { const X* x; X* y; int first, nv, shift; };
  auto row_of = [&](int64_t t) {
    Row r;
    r.x = x + t * a.ldx;
    r.y = y + t * a.ldy;
    r.first = min(D, int((16 - (reinterpret_cast<uintptr_t>(r.y) & 15)) & 15) / SIZE);
    r.shift = APART ? int(reinterpret_cast<uintptr_t>(r.x + r.first) & 15) : 0;
    if (r.shift > r.first * SIZE) r.first = min(D, r.first + N);                         // all of the two vectors' bytes are the row's
    r.nv = max(0, (D - r.first - (APART ? N - r.shift / SIZE : 0)) / N);
    return r;
  };
  uint4 next[NV], more[APART ? NV : 1];
  X next_end[ENDS];
  auto load = [&](const Row& r) {
    const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(r.x + r.first) - r.shift) + at;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (at + i * L < r.nv) {
        next[i] = __ldg(p + i * L);
        if constexpr (APART) more[i] = __ldg(p + i * L + 1);
      }
    const int ends = D - r.nv * N;
#pragma unroll
    for (int i = 0; i < ENDS; ++i) {
      const int e = at + i * L;
      if (e < ends) next_end[i] = r.x[e < r.first ? e : r.nv * N + e];
    }
  };
  Row now, coming = row_of(t0 + mine);
  if (t0 + mine < t1) load(coming);
  {
    float* flat = reinterpret_cast<float*>(pairs);
    auto put = [&](const void* p, float none, int which) {
      auto from = [&](auto w) {
        using W = decltype(w);
        for (int i0 = threadIdx.x; i0 < D; i0 += 8 * blockDim.x) {
          W v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (i0 + j * int(blockDim.x) < D) v[j] = static_cast<const W*>(p)[i0 + j * blockDim.x];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int c = i0 + j * blockDim.x;
            if (c < D) flat[2 * (c % N * columns + c / N) + which] = to_f(v[j]);
          }
        }
        return 0;
      };
      if (p) with_type_device(a.w_type, from);
      else
        for (int i = threadIdx.x; i < N * columns; i += blockDim.x) flat[2 * i + which] = none;
    };
    put(a.weight, 1.0f, 0);
    put(a.bias, 0.0f, 1);
  }
  __syncthreads();
  auto sum = [&](float v, int k) {
    v = lanes_sum<(L < 32 ? L : 32)>(v);
    if constexpr (WARPS > 1) {
      if ((threadIdx.x & 31) == 0) part[k][threadIdx.x >> 5] = v;
      group_sync<L>(mine);
      v = 0.0f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) v += part[k][mine * WARPS + i];
    }
    return v;
  };
  const float share = 1.0f / float(D);
  for (int64_t r0 = t0; r0 < t1; r0 += GROUPS) {
    const int64_t t = r0 + mine;
    now = coming;
    uint4 u[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if constexpr (APART) u[i] = between(next[i], more[i], now.shift);
      else u[i] = next[i];
    }
    float end[ENDS];
    const int n = now.nv > at ? (now.nv - at - 1) / L + 1 : 0, ends = D - now.nv * N;
#pragma unroll
    for (int i = 0; i < ENDS; ++i) end[i] = at + i * L < ends ? to_f(next_end[i]) : 0.0f;
    coming = row_of(t + GROUPS);
    if (t + GROUPS < t1) load(coming);
    f2 s = both(0.0f);
#pragma unroll
    for (int i = 0; i < ENDS; ++i) s = add2(s, pack2(end[i], 0.0f));
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < n)
#pragma unroll
        for (int j = 0; j < N / 2; ++j) s = add2(s, Vec<X>::pair(u[i], j));
    const float mu = sum(add_up(s), 0) * share;
    const f2 minus = both(-mu);
    s = both(0.0f);
#pragma unroll
    for (int i = 0; i < ENDS; ++i) {
      const float d = at + i * L < ends ? end[i] - mu : 0.0f;
      s = fma2(pack2(d, 0.0f), pack2(d, 0.0f), s);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < n)
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
          const f2 d = add2(Vec<X>::pair(u[i], j), minus);
          s = fma2(d, d, s);
        }
    const float rs = rsqrtf(fmaf(sum(add_up(s), 1), share, a.eps));
    if (t >= t1) continue;
    const f2 rs2 = both(rs);
    auto place = [&](int c) { return c % N * columns + c / N; };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (i >= n) break;
      const int v = at + i * L;
      float o[N];
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        // column first + N v + e: with first = N q + f, in the group (f + e) mod N
        const int e0 = now.first + 2 * j, e1 = e0 + 1;
        const float2 p = pairs[place(e0) + v], q = pairs[place(e1) + v];
        unpack2(fma2(mul2(add2(Vec<X>::pair(u[i], j), minus), rs2), pack2(p.x, q.x), pack2(p.y, q.y)), o[2 * j], o[2 * j + 1]);
      }
      __stcs(reinterpret_cast<uint4*>(now.y + now.first) + v, pack_vec<X>(o));
    }
#pragma unroll
    for (int i = 0; i < ENDS; ++i) {
      const int e = at + i * L;
      if (e >= ends) break;
      const int c = e < now.first ? e : now.nv * N + e;
      const float2 p = pairs[place(c)];
      now.y[c] = from_f<X>(fmaf((end[i] - mu) * rs, p.x, p.y));
    }
    if (at == 0) {
      if (a.mean) a.mean[t] = mu;
      if (a.rstd) a.rstd[t] = rs;
    }
  }
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

template <typename X>
__global__ void __launch_bounds__(LONG_TPB) k_norm_long(const X* x, X* y, const __grid_constant__ NormArgs a) {
  __shared__ float sh[LONG_TPB / 32];
  const int64_t t = blockIdx.x;
  const X* row = x + t * a.ldx;
  X* out = y + t * a.ldy;
  float s = 0.0f;
  for (int64_t i = threadIdx.x; i < a.D; i += LONG_TPB) s += to_f(row[i]);
  const float mu = cta_sum(s, sh) / float(a.D);
  s = 0.0f;
  for (int64_t i = threadIdx.x; i < a.D; i += LONG_TPB) {
    const float d = to_f(row[i]) - mu;
    s = fmaf(d, d, s);
  }
  const float r = rsqrtf(cta_sum(s, sh) / float(a.D) + a.eps);
  for (int64_t i = threadIdx.x; i < a.D; i += LONG_TPB)
    out[i] = from_f<X>(fmaf((to_f(row[i]) - mu) * r, parameter(a.weight, a.w_type, i, 1.0f), parameter(a.bias, a.w_type, i, 0.0f)));
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[t] = mu;
    if (a.rstd) a.rstd[t] = r;
  }
}

// ------------------------------------------------------------------------------------------ gradients
struct NormGradArgs {
  int64_t T, D, lddy, ldx, lddx;
  const void* weight;
  int w_type;
  const float *mean, *rstd;
  float *dweight, *dbias, *part;      // part: [CTAs][2][D]
  int accumulate, parts;
  int64_t per;                       // rows per CTA
  int stages, image;
};

// 16 bytes to shared memory, or as many zeros.
__device__ __forceinline__ void fetch(void* to, const void* from, bool any) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(uint32_t(__cvta_generic_to_shared(to))), "l"(from), "r"(any ? 16 : 0) : "memory");
}
__device__ __forceinline__ void fetches_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void fetched(int behind) {        // all but the last `behind` groups of copies have come
  if (behind == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (behind == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// A row that lies anywhere, as the vectors in which its bytes are: L lanes copy them, and it begins (address mod 16) bytes into `to`.  The
// neighbouring rows' bytes may come with it; what is outside the T rows [lo, hi) does not.
inline int image_bytes(int64_t D, int size) { return int((D * size + 15) / 16 + 1) * 16; }
template <typename X, int L> __device__ __forceinline__ void fetch_row(char* to, const X* row, int D, int at, const X* lo, const X* hi) {
  const char* a = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(row) & ~uintptr_t(15));
  const int vecs = int((reinterpret_cast<const char*>(row + D) - a + 15) / 16);
  if (a >= reinterpret_cast<const char*>(lo) && a + 16 * vecs <= reinterpret_cast<const char*>(hi)) {
#pragma unroll 2
    for (int i = at; i < vecs; i += L) fetch(to + 16 * i, a + 16 * i, true);
  } else {                           // the first and the last row
    for (int i = at; i < D; i += L) const_cast<X*>(reinterpret_cast<const X*>(to + (reinterpret_cast<uintptr_t>(row) & 15)))[i] = row[i];
  }
}
template <typename X> __device__ __forceinline__ const X* in_image(const char* image, const X* row) {
  return reinterpret_cast<const X*>(image + (reinterpret_cast<uintptr_t>(row) & 15));
}

// R rows at a time; a thread owns its columns' sums over rows.  The units of x and dy travel through a thread's own places in
// shared memory, a.stages deep, so that nothing waits for them but the thread itself; of rows that lie anywhere, as images that their lanes share.
template <int L> constexpr int GRAD_THREADS = L > NORM_TPB ? L : NORM_TPB;

template <typename X, bool VEC, int L, int NV, int R>
__global__ void __launch_bounds__(GRAD_THREADS<L>, L > NORM_TPB ? 1 : 2) k_norm_grad(const X* dy, const X* x, X* dx, const __grid_constant__ NormGradArgs a) {
  using Un = Unit<X, VEC>;
  constexpr int N = Un::N, PAIRS = NV * N / 2, THREADS = GRAD_THREADS<L>, GROUPS = THREADS / L, WARPS = L / 32, STAGE = R * NV * 2 * THREADS;
  extern __shared__ float4 shared[];         // the ring (or the images), weights, laid out as above; at the end the groups' sums
  __shared__ float part[2][2 * R][THREADS / 32];
  const int D = int(a.D), units = D / N, tid = threadIdx.x, mine = tid / L, at = tid % L;
  const int n = units > at ? (units - at - 1) / L + 1 : 0;
  Un* ring = reinterpret_cast<Un*>(shared);
  char* images = reinterpret_cast<char*>(shared) + mine * (R * 2) * a.image;       // of a group; GROUPS of them for each stage
  const int stage = VEC ? STAGE * 16 : GROUPS * R * 2 * a.image;
  float* pw = reinterpret_cast<float*>(reinterpret_cast<char*>(shared) + a.stages * stage);
  const int64_t t0 = blockIdx.x * a.per, t1 = min(a.T, t0 + a.per);
  constexpr int STEP = GROUPS * R;
  auto row = [&](int64_t r0, int r) { return r0 + r * GROUPS + mine; };
  auto issue = [&](int64_t r0, int slot) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t t = row(r0, r);
      if constexpr (VEC) {
        const int any = t < t1 ? n : 0;
        const X *px = x + t * a.ldx + at * N, *py = dy + t * a.lddy + at * N;
        Un* to = ring + slot * STAGE + r * NV * 2 * THREADS + tid;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          fetch(to + i * 2 * THREADS, i < any ? px + i * L * N : x, i < any);
          fetch(to + (i * 2 + 1) * THREADS, i < any ? py + i * L * N : dy, i < any);
        }
      } else if (t < t1) {
        char* to = images + slot * stage + r * 2 * a.image;
        fetch_row<X, L>(to, x + t * a.ldx, D, at, x, x + (a.T - 1) * a.ldx + D);
        fetch_row<X, L>(to + a.image, dy + t * a.lddy, D, at, dy, dy + (a.T - 1) * a.lddy + D);
      }
    }
    fetches_end();
  };
  float mu[R], rs[R];
  auto statistics = [&](int64_t r0) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t t = row(r0, r);
      mu[r] = t < t1 ? a.mean[t] : 0.0f;
      rs[r] = t < t1 ? a.rstd[t] : 0.0f;
    }
  };
  for (int s = 0; s + 1 < a.stages; ++s) issue(t0 + s * STEP, s);
  statistics(t0);
  put_params<N>(pw, a.weight, a.w_type, 1.0f, D, units);
  f2 dw[PAIRS], db[PAIRS];
#pragma unroll
  for (int k = 0; k < PAIRS; ++k) dw[k] = db[k] = both(0.0f);
  __syncthreads();
  const float share = 1.0f / float(D);
  int flip = 0, slot = 0;
  for (int64_t r0 = t0; r0 < t1; r0 += STEP) {
    if constexpr (VEC) {
      issue(r0 + (a.stages - 1) * STEP, slot == 0 ? a.stages - 1 : slot - 1);
      fetched(a.stages - 1);
    } else {
      fetched(a.stages - 2);
      group_sync<L>(mine);           // the rows have come, and the ones before have been read
      issue(r0 + (a.stages - 1) * STEP, slot == 0 ? a.stages - 1 : slot - 1);
    }
    // x (0) or dy (1) of row r
    auto of = [&](int r, int which) {
      if constexpr (VEC) {
        const Un* from = ring + slot * STAGE + (r * NV * 2 + which) * THREADS + tid;
        return [from](int i) -> const Un& { return from[i * 2 * THREADS]; };
      } else {
        const int64_t t = row(r0, r);
        const X* from = in_image(images + slot * stage + (r * 2 + which) * a.image, which ? dy + t * a.lddy : x + t * a.ldx) + at;
        return [from](int i) { return Un{from[i * L]}; };
      }
    };
    float s[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      f2 s0 = both(0.0f), s1 = s0;
      const int some = VEC || row(r0, r) < t1 ? n : 0;
      const f2 minus = both(-mu[r]), rs2 = both(rs[r]);
      auto gx = of(r, 0), gy = of(r, 1);
      each_pair<X, VEC, NV>(some, [&](int i, int j, int k, bool second) {
        const f2 vx = pair_of<X, VEC>(gx, i, j, second), vy = pair_of<X, VEC>(gy, i, j, second);
        const f2 nn = mul2(add2(vx, minus), rs2), h = mul2(vy, param_pair<N, L>(pw, at, units, k, second));
        s0 = add2(s0, h);
        s1 = fma2(h, nn, s1);
        dw[k] = fma2(vy, nn, dw[k]);
        db[k] = add2(db[k], vy);
      });
      s[2 * r] = add_up(s0);
      s[2 * r + 1] = add_up(s1);
    }
    if (dx) {
#pragma unroll
      for (int j = 0; j < 2 * R; ++j) s[j] = lanes_sum<(L < 32 ? L : 32)>(s[j]);
      if constexpr (WARPS > 1) {
        if ((tid & 31) == 0)
#pragma unroll
          for (int j = 0; j < 2 * R; ++j) part[flip][j][tid >> 5] = s[j];
        group_sync<L>(mine);
#pragma unroll
        for (int j = 0; j < 2 * R; ++j) {
          s[j] = 0.0f;
#pragma unroll
          for (int i = 0; i < WARPS; ++i) s[j] += part[flip][j][mine * WARPS + i];
        }
        flip ^= 1;
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int64_t t = row(r0, r);
        if (t >= t1) continue;
        const f2 minus = both(-mu[r]), rs2 = both(rs[r]), m0 = both(-s[2 * r] * share), m1 = both(-s[2 * r + 1] * share);
        auto gx = of(r, 0), gy = of(r, 1);
        put_pairs<X, VEC, NV, L>(n, dx + t * a.lddx + at * N, [&](int i, int j, int k, bool second) {
          const f2 nn = mul2(add2(pair_of<X, VEC>(gx, i, j, second), minus), rs2);
          return mul2(fma2(nn, m1, fma2(pair_of<X, VEC>(gy, i, j, second), param_pair<N, L>(pw, at, units, k, second), m0)), rs2);
        });
      }
    }
    statistics(r0 + STEP);
    slot = slot + 1 == a.stages ? 0 : slot + 1;
  }
  if (!a.part) return;
  float* out = a.part + int64_t(blockIdx.x) * 2 * D;
  float* sums = GROUPS == 1 ? out : reinterpret_cast<float*>(shared) + mine * 2 * D;
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PAIRS; ++k) {
    float w[2], b[2];
    unpack2(dw[k], w[0], w[1]);
    unpack2(db[k], b[0], b[1]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int c = N == 1 ? at + (2 * k + e) * L : (at + k / (N / 2) * L) * N + k % (N / 2) * 2 + e;
      if (c < D) {
        sums[c] = w[e];
        sums[D + c] = b[e];
      }
    }
  }
  if (GROUPS == 1) return;
  __syncthreads();
  for (int c = tid; c < 2 * D; c += THREADS) {
    float v = 0.0f;
    for (int g = 0; g < GROUPS; ++g) v += reinterpret_cast<const float*>(shared)[g * 2 * D + c];
    out[c] = v;
  }
}

template <typename X>
__global__ void __launch_bounds__(LONG_TPB) k_norm_grad_long(const X* dy, const X* x, X* dx, const __grid_constant__ NormGradArgs a) {
  __shared__ float sh[LONG_TPB / 32];
  float* pw = a.part ? a.part + int64_t(blockIdx.x) * 2 * a.D : nullptr;
  const int64_t t0 = blockIdx.x * a.per, t1 = min(a.T, t0 + a.per);
  for (int64_t t = t0; t < t1; ++t) {
    const X *g = dy + t * a.lddy, *row = x + t * a.ldx;
    const float mu = a.mean[t], r = a.rstd[t];
    float s0 = 0.0f, s1 = 0.0f;
    if (dx) {
      for (int64_t i = threadIdx.x; i < a.D; i += LONG_TPB) {
        const float n = (to_f(row[i]) - mu) * r, h = to_f(g[i]) * parameter(a.weight, a.w_type, i, 1.0f);
        s0 += h;
        s1 = fmaf(h, n, s1);
      }
      s0 = cta_sum(s0, sh) / float(a.D);
      s1 = cta_sum(s1, sh) / float(a.D);
    }
    for (int64_t i = threadIdx.x; i < a.D; i += LONG_TPB) {
      const float n = (to_f(row[i]) - mu) * r, d = to_f(g[i]);
      if (pw) {
        pw[i] = t == t0 ? d * n : fmaf(d, n, pw[i]);
        pw[a.D + i] = t == t0 ? d : pw[a.D + i] + d;
      }
      if (dx) dx[t * a.lddx + i] = from_f<X>(r * (fmaf(d, parameter(a.weight, a.w_type, i, 1.0f), -s0) - n * s1));
    }
  }
}

// The CTAs' sums, 32 columns (of 2 D) per CTA, each by 32 threads in turn.
constexpr int JOIN = 32;
__global__ void __launch_bounds__(32 * JOIN) k_norm_join(const __grid_constant__ NormGradArgs a) {
  __shared__ float sh[JOIN][32];
  const int64_t c = int64_t(blockIdx.x) * 32 + threadIdx.x % 32;
  const int slice = threadIdx.x / 32;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float s = 0.0f;
  if (c < 2 * a.D) {
#pragma unroll 8
    for (int p = slice; p < a.parts; p += JOIN) s += __ldcg(a.part + int64_t(p) * 2 * a.D + c);
  }
  sh[slice][threadIdx.x % 32] = s;
  __syncthreads();
  if (slice || c >= 2 * a.D) return;
  s = sh[0][threadIdx.x];
  for (int i = 1; i < JOIN; ++i) s += sh[i][threadIdx.x];
  float* out = c < a.D ? a.dweight : a.dbias;
  const int64_t i = c < a.D ? c : c - a.D;
  if (out) out[i] = a.accumulate ? out[i] + s : s;
}

// How rows of `units` are shared: by few lanes with many units each where there are many rows, by many lanes where there are few.
struct Shape { int lanes, nv; };

constexpr int MANY_ROWS = 148 * 8, WAVES = 3;

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

constexpr int64_t MOST_PARTS = 1184;
inline int64_t norm_parts(int64_t T, int64_t D) {
  int64_t n = (int64_t(1) << 25) / D;
  if (n > MOST_PARTS) n = MOST_PARTS;
  if (n > T) n = T;
  return n < 1 ? 1 : n;
}

bool unaligned(const void* p, int64_t rows, int64_t ld, int size) { return misaligned(p, 16) || (rows > 1 && ld * size % 16 != 0); }

bool bad_rows(const void* p, int type, int64_t ld, int64_t T, int64_t D) { return (T > 0 && !p) || ld < D || misaligned(p, type_size(type)); }

}  // namespace

extern "C" {

int mv_layer_norm(void* stream, const void* x, int type, int64_t T, int64_t D, int64_t ldx, const void* weight, const void* bias, int w_type,
                  float eps, void* y, int64_t ldy, float* mean, float* rstd) {
  const int64_t lim = int64_t(1) << 31;
  if (!is_value_type(type) || T < 0 || T >= lim || D < 1 || D >= lim || bad_rows(x, type, ldx, T, D) || bad_rows(y, type, ldy, T, D) ||
      (w_type != MV_F32 && w_type != type) || misaligned(weight, type_size(w_type)) || misaligned(bias, type_size(w_type)) || !(eps >= 0.0f) || isinf(eps) ||
      misaligned(mean, 4) || misaligned(rstd, 4))
    return MV_ERR_INVALID_ARG;
  const int size = type_size(type), wsize = type_size(w_type);
  if ((share_bytes(x, T, D, ldx, size, y, T, D, ldy, size) && !(x == y && ldx == ldy)) || (weight && share_bytes(y, T, D, ldy, size, weight, 1, D, D, wsize)) ||
      (bias && share_bytes(y, T, D, ldy, size, bias, 1, D, D, wsize)))
    return MV_ERR_INVALID_ARG;
  if (T == 0) return MV_OK;
  NormArgs a;
  a.T = T; a.D = D; a.ldx = ldx; a.ldy = ldy; a.weight = weight; a.bias = bias; a.w_type = w_type; a.eps = eps; a.mean = mean; a.rstd = rstd;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_type(type, [&](auto xx) {
    using X = decltype(xx);
    const X* xp = static_cast<const X*>(x);
    X* yp = static_cast<X*>(y);
    constexpr int N = Vec<X>::N;
    auto launch = [&](auto* kernel, SmemLimit* limit, int lanes, size_t smem, int64_t resident) {
      const int threads = lanes > 32 ? WIDE_TPB : NORM_TPB;
      const int64_t groups = threads / lanes;
      if (resident * int64_t(smem + 1024) > 227 * 1024) resident = 227 * 1024 / int64_t(smem + 1024);
      // several waves, if a group of lanes has eight rows or more in each CTA (which copies the parameters first)
      int64_t ctas = T / (groups * 8);
      ctas = ctas < resident * 148 ? resident * 148 : ctas > resident * 148 * WAVES ? resident * 148 * WAVES : ctas;
      a.per = ((T + ctas - 1) / ctas + groups - 1) / groups * groups;
      if (smem > 48 * 1024 && !allow_smem(kernel, int(smem), limit)) return int(MV_ERR_CUDA);
      kernel<<<unsigned((T + a.per - 1) / a.per), unsigned(threads), smem, st>>>(xp, yp, a);
      return cuda_ok();
    };
    auto vectors = [&]() {
      Shape s;
      const size_t smem = size_t((D + 3) / 4 * 4) * 8;
      if (smem > 200 * 1024 || !norm_shape(D / N, T, 8, WIDE_TPB, 1, 8, 8, &s)) return -1;
      return with_shape<8, WIDE_TPB, 1, 8, 8, 8>(s, [&](auto lanes, auto nv) {
        constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value;
        static SmemLimit limit;
        return launch(k_norm<X, L, NV>, &limit, L, smem, norm_resident(NV * N, L > 32));
      });
    };
    auto anywhere = [&](auto apart) {
      constexpr bool APART = decltype(apart)::value;
      Shape s;
      const size_t smem = size_t((D + N - 1) / N) * N * 8;
      if (smem > 200 * 1024 || !norm_shape(D / N + 1, T, 8, WIDE_TPB, 4, 4, 8, &s)) return -1;
      return with_shape<8, WIDE_TPB, 4, 4, 8, 8>(s, [&](auto lanes, auto nv) {
        constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value;
        static SmemLimit limit;
        return launch(k_norm_any<X, APART, L, NV>, &limit, L, smem, L > 32 ? 1 : 2);
      });
    };
    const bool vec = D % Vec<X>::N == 0 && !unaligned(x, T, ldx, size) && !unaligned(y, T, ldy, size);
    const bool alike = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15) == 0 && (T == 1 || (ldx - ldy) * size % 16 == 0);
    const int status = vec ? vectors() : alike ? anywhere(std::false_type()) : anywhere(std::true_type());
    if (status != -1) return status;
    k_norm_long<X><<<unsigned(T), LONG_TPB, 0, st>>>(xp, yp, a);
    return cuda_ok();
  });
}

size_t mv_layer_norm_grad_workspace_bytes(int64_t T, int64_t D) {
  const int64_t lim = int64_t(1) << 31;
  if (T < 0 || T >= lim || D < 1 || D >= lim) return 0;
  return align_up(size_t(norm_parts(T, D)) * 2 * size_t(D) * 4, 16);
}

int mv_layer_norm_grad(void* stream, const void* dy, int64_t lddy, const void* x, int64_t ldx, int type, int64_t T, int64_t D,
                       const void* weight, int w_type, const float* mean, const float* rstd, void* dx, int64_t lddx, float* dweight,
                       float* dbias, int accumulate, void* workspace, size_t workspace_bytes) {
  const int64_t lim = int64_t(1) << 31;
  if (!is_value_type(type) || T < 0 || T >= lim || D < 1 || D >= lim || bad_rows(x, type, ldx, T, D) || bad_rows(dy, type, lddy, T, D) ||
      (dx && bad_rows(dx, type, lddx, T, D)) || (w_type != MV_F32 && w_type != type) || misaligned(weight, type_size(w_type)) ||
      (T > 0 && (!mean || !rstd)) || misaligned(mean, 4) || misaligned(rstd, 4) || misaligned(dweight, 4) || misaligned(dbias, 4) ||
      (!dx && !dweight && !dbias) || (accumulate != 0 && accumulate != 1) || misaligned(workspace, 16))
    return MV_ERR_INVALID_ARG;
  const int size = type_size(type), wsize = type_size(w_type);
  if (dx && ((share_bytes(x, T, D, ldx, size, dx, T, D, lddx, size) && !(x == dx && ldx == lddx)) ||
             (share_bytes(dy, T, D, lddy, size, dx, T, D, lddx, size) && !(dy == dx && lddy == lddx)) || (weight && share_bytes(dx, T, D, lddx, size, weight, 1, D, D, wsize))))
    return MV_ERR_INVALID_ARG;
  for (float* p : {dweight, dbias})
    if (p && (share_bytes(x, T, D, ldx, size, p, 1, D, D, 4) || share_bytes(dy, T, D, lddy, size, p, 1, D, D, 4) || (dx && share_bytes(dx, T, D, lddx, size, p, 1, D, D, 4)) ||
              (weight && share_bytes(weight, 1, D, D, wsize, p, 1, D, D, 4))))
      return MV_ERR_INVALID_ARG;
  if (dweight && dbias && share_bytes(dweight, 1, D, D, 4, dbias, 1, D, D, 4)) return MV_ERR_INVALID_ARG;
  if ((dweight || dbias) && (!workspace || workspace_bytes < mv_layer_norm_grad_workspace_bytes(T, D))) return MV_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (T == 0) {
    if (accumulate) return MV_OK;
    for (float* p : {dweight, dbias})
      if (p && cudaMemsetAsync(p, 0, size_t(D) * 4, st) != cudaSuccess) return cuda_ok(), MV_ERR_CUDA;
    return MV_OK;
  }
  NormGradArgs a;
  a.T = T; a.D = D; a.lddy = lddy; a.ldx = ldx; a.lddx = lddx; a.weight = weight; a.w_type = w_type; a.mean = mean; a.rstd = rstd; a.dweight = dweight; a.dbias = dbias;
  a.part = dweight || dbias ? static_cast<float*>(workspace) : nullptr; a.accumulate = accumulate;
  const int64_t most_parts = norm_parts(T, D);
  const int status = with_type(type, [&](auto xx) {
    using X = decltype(xx);
    const X *yp = static_cast<const X*>(dy), *xp = static_cast<const X*>(x);
    X* dxp = static_cast<X*>(dx);
    auto launch = [&](auto vec) {
      constexpr bool VEC = decltype(vec)::value;
      // (images of rows of 32 elements a lane leave room for one CTA only where they are of 4 bytes)
      constexpr int N = Unit<X, VEC>::N, LEAST = VEC ? 1 : 4, LIKED = (VEC || sizeof(X) == 4 ? 16 : 32) / N, MOST = 32 / N;
      Shape s;
      if (!norm_shape(D / N, T, 8, 512, LEAST, LIKED, MOST, &s)) return -1;
      return with_shape<8, 512, LEAST, LIKED, MOST, 8>(s, [&](auto lanes, auto nv) {
        constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value, THREADS = GRAD_THREADS<L>, GROUPS = THREADS / L;
        constexpr int R = NV * N > 16 ? 1 : VEC ? (NV < 4 ? 4 / NV : 1) : (NV < 16 ? 2 : 1);
        a.image = VEC ? 0 : image_bytes(D, size);
        const int64_t stage = VEC ? int64_t(R) * NV * 2 * THREADS * 16 : int64_t(GROUPS) * R * 2 * a.image;
        // Two CTAs of 256 threads with two stages each come before three stages, and more than a few rows for each before more CTAs, whose
        // sums are written and read again.
        int64_t parts = L > NORM_TPB ? 1 : 2;
        const int64_t least_smem = 2 * stage + 4 * D > GROUPS * 8 * D ? 2 * stage + 4 * D : GROUPS * 8 * D;
        if (parts * (least_smem + 2048) > 227 * 1024) parts = 1;
        for (a.stages = 3; a.stages && parts * (a.stages * stage + 4 * D + 2048) > 227 * 1024; --a.stages) {}
        if (a.stages < (VEC ? 1 : 2)) return -1;
        parts *= 148;
        const int64_t few = T * size / 16 > 64 ? T * size / 16 : 64;
        if (parts > few) parts = few;
        if (parts > most_parts) parts = most_parts;
        a.per = ((T + parts - 1) / parts + GROUPS - 1) / GROUPS * GROUPS;
        a.parts = int((T + a.per - 1) / a.per);
        const int64_t turns = (a.per + GROUPS * R - 1) / (GROUPS * R);
        if (a.stages > turns) a.stages = turns > 1 || VEC ? int(turns) : 2;
        size_t smem = size_t(a.stages * stage + 4 * D);
        if (GROUPS > 1 && smem < size_t(GROUPS * 8 * D)) smem = size_t(GROUPS * 8 * D);
        auto* kernel = k_norm_grad<X, VEC, L, NV, R>;
        static SmemLimit limit;
        if (smem > 48 * 1024 && !allow_smem(kernel, int(smem), &limit)) return int(MV_ERR_CUDA);
        kernel<<<unsigned(a.parts), THREADS, smem, st>>>(yp, xp, dxp, a);
        return cuda_ok();
      });
    };
    const bool vec = D % Vec<X>::N == 0 && !unaligned(x, T, ldx, size) && !unaligned(dy, T, lddy, size) && (!dx || !unaligned(dx, T, lddx, size));
    const int status = vec ? launch(std::true_type()) : launch(std::false_type());
    if (status != -1) return status;
    a.per = (T + most_parts - 1) / most_parts;
    a.parts = int((T + a.per - 1) / a.per);
    k_norm_grad_long<X><<<unsigned(a.parts), LONG_TPB, 0, st>>>(yp, xp, dxp, a);
    return cuda_ok();
  });
  if (status != MV_OK || !a.part) return status;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned((2 * D + 31) / 32));
  cfg.blockDim = dim3(32 * JOIN);
  cfg.stream = st;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const bool ok = cudaLaunchKernelEx(&cfg, k_norm_join, a) == cudaSuccess;
  return cuda_ok() == MV_OK && ok ? int(MV_OK) : int(MV_ERR_CUDA);
}

}  // extern "C"
