// mv_norm.cu -- layer norm of rows and its gradients, for sm_100a.

#include "mv_row.cuh"

namespace {

// A row is read once, into registers, by L lanes (L = 32: of one warp or of all warps of a CTA), each with NV units: vectors of 16 bytes where rows
// lie on their boundaries, single elements elsewhere.
template <typename X, bool VEC> struct Unit;
template <typename X> struct Unit<X, true> {
  static constexpr int N = Vec<X>::N;
  uint4 u;
  __device__ __forceinline__ void load(const X* row, int i) { u = __ldcs(reinterpret_cast<const uint4*>(row) + i); }
  __device__ __forceinline__ void clear() { u = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&f)[N]) const {
#pragma unroll
    for (int j = 0; j < N / 2; ++j) unpack2(Vec<X>::pair(u, j), f[2 * j], f[2 * j + 1]);
  }
  __device__ __forceinline__ static void store(X* row, int i, const float (&f)[N]) { __stcs(reinterpret_cast<uint4*>(row) + i, pack_vec<X>(f)); }
};
template <typename X> struct Unit<X, false> {
  static constexpr int N = 1;
  X u;
  __device__ __forceinline__ void load(const X* row, int i) { u = row[i]; }
  __device__ __forceinline__ void clear() { u = from_f<X>(0.0f); }
  __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = to_f(u); }
  __device__ __forceinline__ static void store(X* row, int i, const float (&f)[1]) { row[i] = from_f<X>(f[0]); }
};

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
template <int N> __device__ __forceinline__ void get_params(const float* p, int unit, int units, float (&f)[N]) {
  if constexpr (N == 1) {
    f[0] = p[unit];
  } else {
#pragma unroll
    for (int h = 0; h < N / 4; ++h) {
      const float4 v = reinterpret_cast<const float4*>(p)[h * units + unit];
      f[4 * h] = v.x; f[4 * h + 1] = v.y; f[4 * h + 2] = v.z; f[4 * h + 3] = v.w;
    }
  }
}

struct NormArgs {
  int64_t T, D, ldx, ldy;
  const void *weight, *bias;
  int w_type;
  float eps;
  float *mean, *rstd;
  int64_t per;                       // rows per CTA
};

constexpr int NORM_TPB = 256;

// WIDE: all warps of the CTA share a row, else L lanes have one each.
template <typename X, bool VEC, int L, int NV, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 512 : NORM_TPB) k_norm(const X* x, X* y, const __grid_constant__ NormArgs a) {
  using Un = Unit<X, VEC>;
  constexpr int N = Un::N;
  extern __shared__ float4 params[];         // weights, then biases
  __shared__ float part[2][16];
  const int D = int(a.D), units = D / N;
  float* pw = reinterpret_cast<float*>(params);
  float* pb = pw + (D + 3) / 4 * 4;
  for (int i = threadIdx.x; i < D; i += blockDim.x) {
    pw[place<N>(i, units)] = parameter(a.weight, a.w_type, i, 1.0f);
    pb[place<N>(i, units)] = parameter(a.bias, a.w_type, i, 0.0f);
  }
  const int groups = WIDE ? 1 : NORM_TPB / L, mine = WIDE ? 0 : threadIdx.x / L;
  const int at = WIDE ? threadIdx.x : threadIdx.x % L, span = WIDE ? blockDim.x : L;
  const int64_t t0 = blockIdx.x * a.per, t1 = min(a.T, t0 + a.per);
  Un next[NV], u[NV];
  auto load = [&](int64_t t) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (t < t1 && at + i * span < units) next[i].load(x + t * a.ldx, at + i * span);
      else next[i].clear();
    }
  };
  load(t0 + mine);
  __syncthreads();
  auto sum = [&](float v, int k) {
    v = lanes_sum<L>(v);
    if (WIDE) {
      if ((threadIdx.x & 31) == 0) part[k][threadIdx.x >> 5] = v;
      __syncthreads();
      v = 0.0f;
      for (int i = 0; i < blockDim.x / 32; ++i) v += part[k][i];
    }
    return v;
  };
  const float size = float(D);
  for (int64_t r = t0; r < t1; r += groups) {
    const int64_t t = r + mine;
#pragma unroll
    for (int i = 0; i < NV; ++i) u[i] = next[i];
    load(t + groups);
    float s = 0.0f, f[N];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      u[i].get(f);
      float q = f[0];
#pragma unroll
      for (int e = 1; e < N; ++e) q += f[e];
      s += q;
    }
    const float mu = sum(s, 0) / size;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (at + i * span >= units) break;
      u[i].get(f);
#pragma unroll
      for (int e = 0; e < N; ++e) s = fmaf(f[e] - mu, f[e] - mu, s);
    }
    const float rs = rsqrtf(sum(s, 1) / size + a.eps);
    if (t >= t1) continue;
    X* out = y + t * a.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * span;
      if (v >= units) break;
      u[i].get(f);
      float w[N], b[N];
      get_params<N>(pw, v, units, w);
      get_params<N>(pb, v, units, b);
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = fmaf((f[e] - mu) * rs, w[e], b[e]);
      Un::store(out, v, f);
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
};

// R rows at a time; a thread owns its columns' weights and sums over rows.
template <typename X, bool VEC, int L, int NV, int R, int THREADS>
__global__ void __launch_bounds__(THREADS) k_norm_grad(const X* dy, const X* x, X* dx, const __grid_constant__ NormGradArgs a) {
  using Un = Unit<X, VEC>;
  constexpr int N = Un::N;
  constexpr bool WIDE = THREADS > NORM_TPB;
  extern __shared__ float4 params[];         // weights, laid out as above; at the end the groups' sums, not WIDE
  __shared__ float part[2][2 * R][32];
  const int D = int(a.D), units = D / N;
  float* pw = reinterpret_cast<float*>(params);
  for (int i = threadIdx.x; i < D; i += blockDim.x) pw[place<N>(i, units)] = parameter(a.weight, a.w_type, i, 1.0f);
  const int groups = WIDE ? 1 : NORM_TPB / L, mine = WIDE ? 0 : threadIdx.x / L;
  const int at = WIDE ? threadIdx.x : threadIdx.x % L, span = WIDE ? blockDim.x : L;
  const int64_t t0 = blockIdx.x * a.per, t1 = min(a.T, t0 + a.per);
  float dw[NV][N] = {}, db[NV][N] = {};
  __syncthreads();
  const float size = float(D);
  int flip = 0;
  for (int64_t r0 = t0; r0 < t1; r0 += groups * R) {
    Un ux[R][NV], uy[R][NV];
    float mu[R], rs[R], s[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t t = r0 + r * groups + mine;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (t < t1 && at + i * span < units) {
          ux[r][i].load(x + t * a.ldx, at + i * span);
          uy[r][i].load(dy + t * a.lddy, at + i * span);
        } else {
          ux[r][i].clear();
          uy[r][i].clear();
        }
      }
      mu[r] = t < t1 ? a.mean[t] : 0.0f;
      rs[r] = t < t1 ? a.rstd[t] : 0.0f;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (at + i * span >= units) break;
        float fx[N], fy[N], w[N];
        ux[r][i].get(fx);
        uy[r][i].get(fy);
        get_params<N>(pw, at + i * span, units, w);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float n = (fx[e] - mu[r]) * rs[r], h = fy[e] * w[e];
          s0 += h;
          s1 = fmaf(h, n, s1);
          dw[i][e] = fmaf(fy[e], n, dw[i][e]);
          db[i][e] += fy[e];
        }
      }
      s[2 * r] = s0;
      s[2 * r + 1] = s1;
    }
    if (!dx) continue;
#pragma unroll
    for (int j = 0; j < 2 * R; ++j) s[j] = lanes_sum<L>(s[j]);
    if (WIDE) {
      if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int j = 0; j < 2 * R; ++j) part[flip][j][threadIdx.x >> 5] = s[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 2 * R; ++j) {
        s[j] = 0.0f;
        for (int i = 0; i < blockDim.x / 32; ++i) s[j] += part[flip][j][i];
      }
      flip ^= 1;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t t = r0 + r * groups + mine;
      if (t >= t1) continue;
      const float s0 = s[2 * r] / size, s1 = s[2 * r + 1] / size;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (at + i * span >= units) break;
        float fx[N], fy[N], w[N];
        ux[r][i].get(fx);
        uy[r][i].get(fy);
        get_params<N>(pw, at + i * span, units, w);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float n = (fx[e] - mu[r]) * rs[r];
          fx[e] = rs[r] * (fmaf(fy[e], w[e], -s0) - n * s1);
        }
        Un::store(dx + t * a.lddx, at + i * span, fx);
      }
    }
  }
  if (!a.part) return;
  float* out = a.part + int64_t(blockIdx.x) * 2 * D;
  float* sums = WIDE ? out : pw + mine * 2 * D;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int c = (at + i * span) * N + e;
      if (c < D) {
        sums[c] = dw[i][e];
        sums[D + c] = db[i][e];
      }
    }
  if (WIDE) return;
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * D; c += NORM_TPB) {
    float v = 0.0f;
    for (int g = 0; g < groups; ++g) v += pw[g * 2 * D + c];
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

// The CTAs' sums, 32 columns (of 2 D) per CTA, each by eight threads in turn.
constexpr int JOIN = 8;
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
struct Shape {
  int lanes, nv, threads;            // lanes per row, units of each, threads per CTA; more than 32 lanes: a CTA per row
  bool wide() const { return lanes > 32; }
  int groups() const { return wide() ? 1 : threads / lanes; }
};

constexpr int MANY_ROWS = 148 * 8;

inline int pow2_at_least(int64_t n) {
  int p = 1;
  while (p < n) p *= 2;
  return p;
}

// least and most units per lane: powers of two
inline bool norm_shape(int64_t units, int64_t T, int least_lanes, int most_lanes, int least, int most, Shape* s) {
  if (units > int64_t(most_lanes) * most) return false;
  int64_t lanes = pow2_at_least((units + (T >= MANY_ROWS ? most : least) - 1) / (T >= MANY_ROWS ? most : least));
  if (lanes < least_lanes) lanes = least_lanes;
  if (lanes > most_lanes) lanes = most_lanes;
  s->nv = pow2_at_least((units + lanes - 1) / lanes);
  if (s->nv < least) s->nv = least;
  if (lanes > 32) lanes = (((units + s->nv - 1) / s->nv) + 31) / 32 * 32;
  s->lanes = int(lanes);
  s->threads = s->wide() ? s->lanes : NORM_TPB;
  return true;
}

template <int I> using Int = std::integral_constant<int, I>;
// Calls f with the lanes (0: more than 32) and the units per lane as constants.
template <typename F> int with_lanes(const Shape& s, F&& f) {
  return s.lanes == 8 ? f(Int<8>()) : s.lanes == 16 ? f(Int<16>()) : s.wide() ? f(Int<0>()) : f(Int<32>());
}
template <int LEAST, int MOST, typename F> int with_units(int nv, F&& f) {
  if constexpr (LEAST >= MOST) return f(Int<MOST>());
  else return nv <= LEAST ? f(Int<LEAST>()) : with_units<LEAST * 2, MOST>(nv, f);
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
    auto launch = [&](auto vec) {
      constexpr bool VEC = decltype(vec)::value;
      constexpr int N = Unit<X, VEC>::N, LEAST = VEC ? 1 : 4, MOST = VEC ? 8 : 32;
      Shape s;
      const size_t smem = size_t((D + 3) / 4 * 4) * 8;
      if (smem > 200 * 1024 || !norm_shape(D / N, T, VEC ? 8 : 32, 512, LEAST, MOST, &s)) return -1;
      const int64_t waves = int64_t(148) * (2048 / s.threads) * 2, groups = s.groups();
      a.per = ((T + waves - 1) / waves + groups - 1) / groups * groups;
      return with_lanes(s, [&](auto lanes) {
        return with_units<LEAST, MOST>(s.nv, [&](auto nv) {
          constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value;
          auto* kernel = k_norm<X, VEC, L ? L : 32, NV, L == 0>;
          static SmemLimit limit;
          if (smem > 48 * 1024 && !allow_smem(kernel, int(smem), &limit)) return int(MV_ERR_CUDA);
          kernel<<<unsigned((T + a.per - 1) / a.per), s.threads, smem, st>>>(xp, yp, a);
          return cuda_ok();
        });
      });
    };
    const bool vec = D % Vec<X>::N == 0 && !unaligned(x, T, ldx, size) && !unaligned(y, T, ldy, size);
    const int status = vec ? launch(std::true_type()) : launch(std::false_type());
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
      constexpr int N = Unit<X, VEC>::N, LEAST = VEC ? 1 : 4, MOST = 16 / N;
      Shape s;
      if (!norm_shape(D / N, T, VEC ? 8 : 32, 1024, LEAST, MOST, &s)) return -1;
      const int64_t groups = s.groups();
      int64_t parts = int64_t(148) * (s.threads > 512 ? 1 : s.threads >= 256 ? 768 / s.threads : 6);
      if (parts > most_parts) parts = most_parts;
      a.per = ((T + parts - 1) / parts + groups - 1) / groups * groups;
      a.parts = int((T + a.per - 1) / a.per);
      const size_t smem = size_t(s.wide() || !a.part ? 1 : groups * 2) * D * 4;
      return with_lanes(s, [&](auto lanes) {
        return with_units<LEAST, MOST>(s.nv, [&](auto nv) {
          constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value, R = VEC ? (NV < 4 ? 4 / NV : 1) : (NV < 16 ? 2 : 1);
          auto* kernel = L ? k_norm_grad<X, VEC, L ? L : 32, NV, R, NORM_TPB> : s.threads <= 512 ? k_norm_grad<X, VEC, 32, NV, R, 512> : k_norm_grad<X, VEC, 32, NV, 1, 1024>;
          static SmemLimit limit;
          if (smem > 48 * 1024 && !allow_smem(kernel, int(smem), &limit)) return int(MV_ERR_CUDA);
          kernel<<<unsigned(a.parts), s.threads, smem, st>>>(yp, xp, dxp, a);
          return cuda_ok();
        });
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
