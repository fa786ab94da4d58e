// mv_token.cu -- log probabilities of given tokens with entropy and alternatives, and their gradient, for sm_100a.
//
// With z = c x, m the row's largest logit and t = (x - m) c log2(e):  s = sum 2^t,  lse = c m + log s,
// H = log s - ln 2 (sum 2^t t) / s.  A masked logit (-inf) has 2^t = 0 and must not multiply its t, so t is kept above
// a finite floor.  The difference x - m is formed before it is scaled: c m alone may overflow (a row of the type's
// lowest value).
#include "mv_lm.cuh"

#include <math.h>

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float T_FLOOR = -1.0e30f;
constexpr int TPB = 256;

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

template <typename F> __device__ float block_reduce(float x, float* sh, F f) {
  for (int o = 16; o; o >>= 1) x = f(x, __shfl_xor_sync(0xffffffffu, x, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
  __syncthreads();
  x = sh[0];
  for (int i = 1; i < TPB / 32; ++i) x = f(x, sh[i]);
  return x;
}

template <typename X>
__global__ void __launch_bounds__(TPB) k_token_logprob(const X* __restrict__ logits, int64_t V, int64_t ld, const void* __restrict__ targets, int id_type,
                                                        float scale, int k, float* logprob, float* entropy, float* lse, float* top_logprob,
                                                        int32_t* top_id) {
  __shared__ float sh[TPB / 32];
  __shared__ float s_v[TPB / 32];
  __shared__ int32_t s_i[TPB / 32];
  const int64_t t = blockIdx.x;
  const X* x = logits + t * ld;
  float m = -INFINITY;
  for (int64_t j = threadIdx.x; j < V; j += TPB) m = max_nan(m, to_f(x[j]));
  m = block_reduce(m, sh, [](float a, float b) { return max_nan(a, b); });
  const float ref = m == -INFINITY ? 0.0f : m;
  float s = 0.0f, st = 0.0f;
  for (int64_t j = threadIdx.x; j < V; j += TPB) {
    const float u = max_nan((to_f(x[j]) - ref) * (scale * LOG2E), T_FLOOR);
    const float e = exp2f(u);
    s += e;
    st = fmaf(e, u, st);
  }
  s = block_reduce(s, sh, [](float a, float b) { return a + b; });
  st = block_reduce(st, sh, [](float a, float b) { return a + b; });
  const float l = s == 0.0f ? -INFINITY : fmaf(scale, ref, logf(s));
  if (threadIdx.x == 0) {
    if (lse) lse[t] = l;
    if (entropy) entropy[t] = s == 0.0f ? 0.0f : logf(s) - LN2 * (st / s);
    if (logprob) {
      const int64_t y = load_id(targets, id_type, t, V);
      logprob[t] = y < 0 ? 0.0f : s == 0.0f ? -INFINITY : (to_f(x[y]) - ref) * scale - logf(s);
    }
  }
  // the next alternative is the largest logit after the last one in (value descending, index ascending) order
  float pv = INFINITY;
  int32_t pi = -1;
  for (int r = 0; r < k; ++r) {
    float bv = -INFINITY;
    int32_t bi = -1;
    for (int64_t j = threadIdx.x; j < V; j += TPB) {
      const float v = to_f(x[j]);
      const bool after = v < pv || (v == pv && j > pi);
      if (after && (bi < 0 || v > bv)) { bv = v; bi = int32_t(j); }
    }
    for (int o = 16; o; o >>= 1) {
      const float ov = __shfl_xor_sync(0xffffffffu, bv, o);
      const int32_t oi = __shfl_xor_sync(0xffffffffu, bi, o);
      if (oi >= 0 && (bi < 0 || ov > bv || (ov == bv && oi < bi))) { bv = ov; bi = oi; }
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) { s_v[threadIdx.x >> 5] = bv; s_i[threadIdx.x >> 5] = bi; }
    __syncthreads();
    bv = s_v[0]; bi = s_i[0];
    for (int w = 1; w < TPB / 32; ++w)
      if (s_i[w] >= 0 && (bi < 0 || s_v[w] > bv || (s_v[w] == bv && s_i[w] < bi))) { bv = s_v[w]; bi = s_i[w]; }
    if (threadIdx.x == 0) {
      if (top_id) top_id[t * k + r] = bi;
      if (top_logprob) top_logprob[t * k + r] = isnan(l) ? l : bi < 0 || bv == -INFINITY ? -INFINITY : (bv - ref) * scale - logf(s);
    }
    if (bi >= 0) { pv = bv; pi = bi; } else { pv = -INFINITY; pi = 0x7fffffff; }
  }
}

template <typename X>
__global__ void __launch_bounds__(TPB) k_token_grad(const X* logits, int64_t V, int64_t ld, const void* __restrict__ targets, int id_type, float scale,
                                                     const float* __restrict__ lse, const float* __restrict__ entropy, const float* __restrict__ g_logprob,
                                                     const float* __restrict__ g_entropy, X* dlogits, int64_t ldg) {
  const int64_t t = blockIdx.x;
  const X* x = logits + t * ld;
  X* dx = dlogits + t * ldg;
  const int64_t y = targets ? load_id(targets, id_type, t, V) : -1;
  const float l = lse[t];
  const float g1 = y >= 0 && g_logprob ? g_logprob[t] : 0.0f;
  const float g2 = g_entropy ? g_entropy[t] : 0.0f;
  const bool none = (g1 == 0.0f && g2 == 0.0f) || l == -INFINITY;
  const float a = g1 + (g2 == 0.0f ? 0.0f : g2 * entropy[t]);
  for (int64_t j = threadIdx.x; j < V; j += TPB) {
    float d = 0.0f;
    if (!none) {
      const float lp = max_nan(fmaf(to_f(x[j]), scale, -l), T_FLOOR);
      const float p = exp2f(lp * LOG2E);
      d = -p * fmaf(g2, lp, a);
      if (j == y) d += g1;
      d *= scale;
    }
    dx[j] = from_f<X>(d);
  }
}

}  // namespace

extern "C" {

int mv_token_logprob(void* stream, const void* logits, int type, int64_t T, int64_t V, int64_t ld, const void* targets, int id_type,
                     float scale, int k, float* logprob, float* entropy, float* lse, float* top_logprob, int32_t* top_id) {
  const int64_t lim = int64_t(1) << 31;
  if (!is_value_type(type) || T < 0 || T >= lim || V < 1 || V >= lim || ld < V || !(scale > 0.0f) || isinf(scale) || k < 0 || k > MV_TOP_MAX ||
      (T > 0 && !logits) || (logprob && T > 0 && !targets) || (targets && !is_id_type(id_type)) || misaligned(logits, type_size(type)) ||
      (targets && misaligned(targets, type_size(id_type))) || misaligned(logprob, 4) || misaligned(entropy, 4) || misaligned(lse, 4) ||
      misaligned(top_logprob, 4) || misaligned(top_id, 4))
    return MV_ERR_INVALID_ARG;
  if (T == 0) return MV_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!top_logprob && !top_id) k = 0;
  return with_type(type, [&](auto x) {
    using X = decltype(x);
    k_token_logprob<X><<<unsigned(T), TPB, 0, st>>>(static_cast<const X*>(logits), V, ld, targets, id_type, scale, k, logprob, entropy, lse,
                                                     top_logprob, top_id);
    return cuda_ok();
  });
}

int mv_token_logprob_grad(void* stream, const void* logits, int type, int64_t T, int64_t V, int64_t ld, const void* targets,
                          int id_type, float scale, const float* lse, const float* entropy, const float* g_logprob,
                          const float* g_entropy, void* dlogits, int64_t ldg) {
  const int64_t lim = int64_t(1) << 31;
  if (!is_value_type(type) || T < 0 || T >= lim || V < 1 || V >= lim || ld < V || ldg < V || !(scale > 0.0f) || isinf(scale) ||
      (T > 0 && (!logits || !lse || !dlogits)) || (!g_logprob && !g_entropy) || (g_logprob && T > 0 && !targets) ||
      (g_entropy && T > 0 && !entropy) || (targets && !is_id_type(id_type)) || misaligned(logits, type_size(type)) ||
      misaligned(dlogits, type_size(type)) || (targets && misaligned(targets, type_size(id_type))) || misaligned(lse, 4) ||
      misaligned(entropy, 4) || misaligned(g_logprob, 4) || misaligned(g_entropy, 4))
    return MV_ERR_INVALID_ARG;
  if (T == 0) return MV_OK;
  // in place element by element, or apart
  const char *a = static_cast<const char*>(logits), *b = static_cast<const char*>(dlogits);
  const int64_t na = ((T - 1) * ld + V) * type_size(type), nb = ((T - 1) * ldg + V) * type_size(type);
  if (a < b + nb && b < a + na && !(a == b && ld == ldg)) return MV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_type(type, [&](auto x) {
    using X = decltype(x);
    k_token_grad<X><<<unsigned(T), TPB, 0, st>>>(static_cast<const X*>(logits), V, ld, targets, id_type, scale, lse, entropy, g_logprob, g_entropy,
                                                  static_cast<X*>(dlogits), ldg);
    return cuda_ok();
  });
}

}  // extern "C"
