// mv_distill.cu -- divergence from a teacher that is known by its largest log probabilities, and its gradient, for sm_100a.
//
// The exponentials and their sums are in mv_row.cuh.

#include "mv_row.cuh"

namespace {

struct Teacher {
  const float* top;                  // [T, k]
  const void* id;
  int id_type, k, rest;
};

// What a row's alternatives add up to, in 64 bits (1 - sum q is a small difference).
struct Mass {
  double scale, rest, all;           // q = scale exp(a - shift), r, M = sum q + r
  float shift;
  bool any, bad;                     // an alternative; a NaN or +inf
};

// The alternative j of row t: its log probability, -inf and column -1 where there is none.
__device__ __forceinline__ float alternative(const Teacher& h, int64_t t, int j, int64_t V, int64_t& col) {
  col = load_id(h.id, h.id_type, t * h.k + j, V);
  return col < 0 ? -INFINITY : h.top[t * h.k + j];
}

// For every lane of a warp.
__device__ __forceinline__ Mass mass_of_row(const Teacher& h, int64_t t, int64_t V) {
  const int lane = threadIdx.x & 31;
  float m = -INFINITY;
  bool any = false, bad = false;
  for (int j = lane; j < h.k; j += 32) {
    int64_t c;
    const float a = alternative(h, t, j, V, c);
    any |= c >= 0 && (h.rest || a != -INFINITY);
    bad |= !(a < INFINITY);
    m = fmaxf(m, a);
  }
  Mass s;
  s.any = __any_sync(0xffffffffu, any);
  s.bad = __any_sync(0xffffffffu, bad);
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  s.shift = h.rest || m == -INFINITY ? 0.0f : m;
  double q = 0.0;
  for (int j = lane; j < h.k; j += 32) {
    int64_t c;
    const float a = alternative(h, t, j, V, c);
    if (a != -INFINITY) q += exp(double(a) - double(s.shift));
  }
  for (int o = 16; o; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
  s.scale = h.rest ? 1.0 : 1.0 / q;
  s.rest = h.rest ? fmax(0.0, 1.0 - q) : 0.0;
  s.all = h.rest ? q + s.rest : 1.0;
  return s;
}

struct DistillArgs {
  int64_t V, ld;
  Teacher h;
  float scale;
  float *kl, *lse, *log_rest;
};

constexpr int WINDOW = 65536;        // columns whose listed tokens are marked at a time

template <typename X, int TPB>
__global__ void __launch_bounds__(TPB) k_distill(const X* __restrict__ logits, const __grid_constant__ DistillArgs a) {
  __shared__ uint32_t mark[WINDOW / 32];
  __shared__ float sh[TPB / 32];
  __shared__ double shd[2][TPB / 32];
  const int64_t t = blockIdx.x;
  const X* row = logits + t * a.ld;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  float m = -INFINITY;
  for (int64_t c = threadIdx.x; c < a.V; c += TPB) m = max_nan(m, to_f(row[c]));
  for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) sh[w] = m;
  __syncthreads();
  for (int i = 0; i < TPB / 32; ++i) m = max_nan(m, sh[i]);
  const float ref = m == -INFINITY ? 0.0f : m;
  double rest = 0.0, listed = 0.0;
  for (int64_t c0 = 0; c0 < a.V; c0 += WINDOW) {
    const int64_t c1 = min(a.V, c0 + WINDOW);
    __syncthreads();
    for (int i = threadIdx.x; i < WINDOW / 32; i += TPB) mark[i] = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < a.h.k; j += TPB) {
      int64_t c;
      alternative(a.h, t, j, a.V, c);
      if (c >= c0 && c < c1) atomicOr(&mark[(c - c0) / 32], 1u << ((c - c0) & 31));
    }
    __syncthreads();
    for (int64_t c = c0 + threadIdx.x; c < c1; c += TPB) {
      const double e = exp2_fast(distance(to_f(row[c]), ref, a.scale) * LOG2E);
      (mark[(c - c0) / 32] >> ((c - c0) & 31) & 1u ? listed : rest) += e;
    }
  }
  for (int o = 16; o; o >>= 1) {
    rest += __shfl_xor_sync(0xffffffffu, rest, o);
    listed += __shfl_xor_sync(0xffffffffu, listed, o);
  }
  if (lane == 0) { shd[0][w] = rest; shd[1][w] = listed; }
  __syncthreads();
  if (w) return;
  rest = listed = 0.0;
  for (int i = 0; i < TPB / 32; ++i) { rest += shd[0][i]; listed += shd[1][i]; }
  const bool nan = !(m < INFINITY);
  const double ls = log(rest + listed), lr = log(rest) - ls;
  const Mass s = mass_of_row(a.h, t, a.V);
  double kl = 0.0;
  if (s.any)
    for (int j = lane; j < a.h.k; j += 32) {
      int64_t c;
      const float l = alternative(a.h, t, j, a.V, c);
      if (l == -INFINITY) continue;
      const double logq = double(l) - double(s.shift) + log(s.scale), q = exp(logq);
      if (q > 0.0) kl += q * (logq - (double(distance(to_f(row[c]), ref, a.scale)) - ls));
    }
  for (int o = 16; o; o >>= 1) kl += __shfl_xor_sync(0xffffffffu, kl, o);
  if (lane == 0) {
    if (s.any && s.rest > 0.0) kl += s.rest * (log(s.rest) - lr);
    const bool empty = m == -INFINITY;
    if (a.kl) a.kl[t] = nan || s.bad ? NAN : !s.any ? 0.0f : empty ? INFINITY : float(kl);
    if (a.lse) a.lse[t] = nan ? NAN : empty ? -INFINITY : fmaf(a.scale, ref, float(ls));
    if (a.log_rest) a.log_rest[t] = nan ? NAN : empty ? -INFINITY : float(lr);
  }
}

struct DistillGradArgs {
  int64_t V, ld, ldg;
  Teacher h;
  float scale;
  const float *lse, *log_rest, *g;
};

template <typename X, int TPB>
__global__ void __launch_bounds__(TPB) k_distill_grad(const X* logits, X* dlogits, const __grid_constant__ DistillGradArgs a) {
  __shared__ float sh[4];
  __shared__ int64_t s_id[MV_TEACHER_MAX];
  __shared__ float s_q[MV_TEACHER_MAX], s_x[MV_TEACHER_MAX];
  const int64_t t = blockIdx.x;
  const X* x = logits + t * a.ld;
  X* dx = dlogits + t * a.ldg;
  if (threadIdx.x < 32) {
    const Mass s = mass_of_row(a.h, t, a.V);
    const float l = a.lse[t], g = a.g[t];
    for (int j = threadIdx.x; j < a.h.k; j += 32) {
      int64_t c;
      const float v = alternative(a.h, t, j, a.V, c);
      s_id[j] = c;
      s_q[j] = float(exp(double(v) - double(s.shift)) * s.scale);
      s_x[j] = c >= 0 ? to_f(x[c]) : 0.0f;
    }
    if (threadIdx.x == 0) {
      const bool none = !s.any || g == 0.0f || l == -INFINITY;
      float ratio = 0.0f;
      if (a.h.rest && s.rest > 0.0) ratio = a.log_rest[t] == -INFINITY ? float(s.all) : float(exp(log(s.rest) - double(a.log_rest[t])));
      sh[0] = none ? 0.0f : a.scale * g;
      sh[1] = s.bad ? NAN : float(s.all);
      sh[2] = s.bad ? NAN : float(s.all - double(ratio));
      sh[3] = l;
    }
  }
  __syncthreads();
  const float f = sh[0], all = sh[1], other = sh[2], l = sh[3];
  for (int64_t c = threadIdx.x; c < a.V; c += TPB) {
    bool listed = false;
    for (int j = 0; j < a.h.k && !listed; ++j) listed = s_id[j] == c;
    if (!listed) dx[c] = from_f<X>(f == 0.0f ? 0.0f : f * other * expf(min_nan(fmaf(to_f(x[c]), a.scale, -l), 0.0f)));
  }
  for (int j = threadIdx.x; j < a.h.k; j += TPB) {
    const int64_t c = s_id[j];
    if (c < 0) continue;
    float q = 0.0f;
    bool first = true;
    for (int i = 0; i < a.h.k; ++i)
      if (s_id[i] == c) {
        first &= i >= j;
        q += s_q[i];
      }
    if (first) dx[c] = from_f<X>(f == 0.0f ? 0.0f : f * (all * expf(min_nan(fmaf(s_x[j], a.scale, -l), 0.0f)) - q));
  }
}

bool bad_list(const float* top, const void* id, int id_type, int k, int64_t T) {
  return k < 1 || k > MV_TEACHER_MAX || !is_id_type(id_type) || (T > 0 && (!top || !id)) || misaligned(top, 4) || misaligned(id, type_size(id_type));
}

}  // namespace

extern "C" {

int mv_distill(void* stream, const void* logits, int type, int64_t T, int64_t V, int64_t ld, const float* top_logprob, const void* top_id,
               int id_type, int k, int rest, float scale, float* kl, float* lse, float* log_rest) {
  const int64_t lim = int64_t(1) << 31;
  if (!is_value_type(type) || T < 0 || T >= lim || V < 1 || V >= lim || ld < V || !(scale > 0.0f) || isinf(scale) || (T > 0 && !logits) ||
      misaligned(logits, type_size(type)) || bad_list(top_logprob, top_id, id_type, k, T) || (rest != 0 && rest != 1) || (log_rest && !rest) ||
      misaligned(kl, 4) || misaligned(lse, 4) || misaligned(log_rest, 4))
    return MV_ERR_INVALID_ARG;
  if (T == 0) return MV_OK;
  DistillArgs a;
  a.V = V; a.ld = ld; a.h = {top_logprob, top_id, id_type, k, rest}; a.scale = scale; a.kl = kl; a.lse = lse; a.log_rest = log_rest;
  return with_type(type, [&](auto x) {
    using X = decltype(x);
    k_distill<X, 256><<<unsigned(T), 256, 0, static_cast<cudaStream_t>(stream)>>>(static_cast<const X*>(logits), a);
    return cuda_ok();
  });
}

int mv_distill_grad(void* stream, const void* logits, int type, int64_t T, int64_t V, int64_t ld, const float* top_logprob,
                    const void* top_id, int id_type, int k, float scale, const float* lse, const float* log_rest, const float* g,
                    void* dlogits, int64_t ldg) {
  const int64_t lim = int64_t(1) << 31;
  if (!is_value_type(type) || T < 0 || T >= lim || V < 1 || V >= lim || ld < V || ldg < V || !(scale > 0.0f) || isinf(scale) ||
      (T > 0 && (!logits || !dlogits || !lse || !g)) || misaligned(logits, type_size(type)) || misaligned(dlogits, type_size(type)) ||
      bad_list(top_logprob, top_id, id_type, k, T) || misaligned(lse, 4) || misaligned(log_rest, 4) || misaligned(g, 4))
    return MV_ERR_INVALID_ARG;
  if (T == 0) return MV_OK;
  const int size = type_size(type);
  if ((share_bytes(logits, T, V, ld, size, dlogits, T, V, ldg, size) && !(logits == dlogits && ld == ldg)) ||
      share_bytes(dlogits, T, V, ldg, size, top_logprob, T, k, k, 4) || share_bytes(dlogits, T, V, ldg, size, top_id, T, k, k, type_size(id_type)))
    return MV_ERR_INVALID_ARG;
  DistillGradArgs a;
  a.V = V; a.ld = ld; a.ldg = ldg; a.h = {top_logprob, top_id, id_type, k, log_rest ? 1 : 0}; a.scale = scale; a.lse = lse; a.log_rest = log_rest; a.g = g;
  return with_type(type, [&](auto x) {
    using X = decltype(x);
    k_distill_grad<X, 256><<<unsigned(T), 256, 0, static_cast<cudaStream_t>(stream)>>>(static_cast<const X*>(logits), static_cast<X*>(dlogits), a);
    return cuda_ok();
  });
}

}  // extern "C"
