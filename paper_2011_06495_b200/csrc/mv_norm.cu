// mv_norm.cu -- layer norm of rows and its gradients, for sm_100a.

#include "mv_lm.cuh"

#include <math.h>

namespace {

struct NormArgs {
  int64_t T, D, ldx, ldy;
  float eps;
  float *mean, *rstd;
};

constexpr int TPB = 256;

// The sum of a value over the CTA, for every thread.
__device__ __forceinline__ float cta_sum(float v, float* sh) {
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0f;
  for (int i = 0; i < TPB / 32; ++i) v += sh[i];
  return v;
}

template <typename X, typename W>
__global__ void __launch_bounds__(TPB) k_norm(const X* x, const W* weight, const W* bias, X* y, const __grid_constant__ NormArgs a) {
  __shared__ float sh[TPB / 32];
  const int64_t t = blockIdx.x;
  const X* row = x + t * a.ldx;
  X* out = y + t * a.ldy;
  float s = 0.0f;
  for (int64_t i = threadIdx.x; i < a.D; i += TPB) s += to_f(row[i]);
  const float mu = cta_sum(s, sh) / float(a.D);
  s = 0.0f;
  for (int64_t i = threadIdx.x; i < a.D; i += TPB) {
    const float d = to_f(row[i]) - mu;
    s = fmaf(d, d, s);
  }
  const float r = 1.0f / sqrtf(cta_sum(s, sh) / float(a.D) + a.eps);
  for (int64_t i = threadIdx.x; i < a.D; i += TPB)
    out[i] = from_f<X>(fmaf((to_f(row[i]) - mu) * r, weight ? to_f(weight[i]) : 1.0f, bias ? to_f(bias[i]) : 0.0f));
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[t] = mu;
    if (a.rstd) a.rstd[t] = r;
  }
}

struct NormGradArgs {
  int64_t T, D, lddy, ldx, lddx;
  const float *mean, *rstd;
  float *dweight, *dbias, *part;      // part: [CTAs][2][D]
  int accumulate, parts;
};

inline int64_t norm_parts(int64_t T, int64_t D) {
  int64_t n = (int64_t(1) << 24) / D;
  if (n > 592) n = 592;
  if (n > T) n = T;
  return n < 1 ? 1 : n;
}

template <typename X, typename W>
__global__ void __launch_bounds__(TPB) k_norm_grad(const X* dy, const X* x, const W* weight, X* dx, const __grid_constant__ NormGradArgs a) {
  __shared__ float sh[TPB / 32];
  float* pw = a.part + int64_t(blockIdx.x) * 2 * a.D;
  float* pb = pw + a.D;
  bool first = true;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const X *g = dy + t * a.lddy, *row = x + t * a.ldx;
    const float mu = a.mean[t], r = a.rstd[t];
    float s0 = 0.0f, s1 = 0.0f;
    if (dx) {
      for (int64_t i = threadIdx.x; i < a.D; i += TPB) {
        const float n = (to_f(row[i]) - mu) * r, h = to_f(g[i]) * (weight ? to_f(weight[i]) : 1.0f);
        s0 += h;
        s1 = fmaf(h, n, s1);
      }
      s0 = cta_sum(s0, sh) / float(a.D);
      s1 = cta_sum(s1, sh) / float(a.D);
    }
    for (int64_t i = threadIdx.x; i < a.D; i += TPB) {
      const float n = (to_f(row[i]) - mu) * r, d = to_f(g[i]), h = d * (weight ? to_f(weight[i]) : 1.0f);
      if (a.dweight) pw[i] = first ? d * n : fmaf(d, n, pw[i]);
      if (a.dbias) pb[i] = first ? d : pb[i] + d;
      if (dx) dx[t * a.lddx + i] = from_f<X>(r * (h - s0 - n * s1));
    }
    first = false;
  }
}

__global__ void __launch_bounds__(TPB) k_norm_join(const __grid_constant__ NormGradArgs a) {
  const int64_t i = int64_t(blockIdx.x) * TPB + threadIdx.x;
  if (i >= a.D) return;
  for (int j = 0; j < 2; ++j) {
    float* out = j ? a.dbias : a.dweight;
    if (!out) continue;
    float s = 0.0f;
    for (int p = 0; p < a.parts; ++p) s += a.part[(int64_t(p) * 2 + j) * a.D + i];
    out[i] = a.accumulate ? out[i] + s : s;
  }
}

// Calls f with null pointers of the element type of the rows and of the parameters.
template <typename F> int with_types(int type, int w_type, F&& f) {
  return with_type(type, [&](auto x) {
    using X = decltype(x);
    if (w_type == MV_F32) return f(static_cast<X*>(nullptr), static_cast<float*>(nullptr));
    return f(static_cast<X*>(nullptr), static_cast<X*>(nullptr));
  });
}

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
  a.T = T; a.D = D; a.ldx = ldx; a.ldy = ldy; a.eps = eps; a.mean = mean; a.rstd = rstd;
  return with_types(type, w_type, [&](auto* xp, auto* wp) {
    using X = std::remove_pointer_t<decltype(xp)>;
    using W = std::remove_pointer_t<decltype(wp)>;
    k_norm<X, W><<<unsigned(T), TPB, 0, static_cast<cudaStream_t>(stream)>>>(static_cast<const X*>(x), static_cast<const W*>(weight),
                                                                            static_cast<const W*>(bias), static_cast<X*>(y), a);
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
  a.T = T; a.D = D; a.lddy = lddy; a.ldx = ldx; a.lddx = lddx; a.mean = mean; a.rstd = rstd; a.dweight = dweight; a.dbias = dbias;
  a.part = static_cast<float*>(workspace); a.accumulate = accumulate; a.parts = int(norm_parts(T, D));
  return with_types(type, w_type, [&](auto* xp, auto* wp) {
    using X = std::remove_pointer_t<decltype(xp)>;
    using W = std::remove_pointer_t<decltype(wp)>;
    k_norm_grad<X, W><<<unsigned(a.parts), TPB, 0, st>>>(static_cast<const X*>(dy), static_cast<const X*>(x), static_cast<const W*>(weight), static_cast<X*>(dx), a);
    if (dweight || dbias) k_norm_join<<<unsigned((D + TPB - 1) / TPB), TPB, 0, st>>>(a);
    return cuda_ok();
  });
}

}  // extern "C"
