// mv_sample.cu -- one token per row from softmax(scale * logits), cut to the top k, the top p and the min p, for sm_100a.
//
// Whether a token stays, and which one is drawn, hangs on where a sum of weights passes a limit; with 10^5 tokens the borders between
// them lie 10^-5 of the sum apart and less, so weights are formed in 64 bits.  They are added as whole numbers, the largest being 2^61 / V
// (V rounded up to a power of two): sums are exact and do not depend on the order in which they are formed.

#include "mv_row.cuh"

namespace {

typedef unsigned long long u64;

struct SampleArgs {
  int64_t V, ld;
  const float *u, *scale, *top_p, *min_p;
  const int32_t* top_k;
  double unit;                       // whole numbers that the largest weight is
  void* token;
  int id_type;
  float* logprob;
};

// The order of the logits as that of 32-bit numbers: larger is earlier; +0 and -0 are one value.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t h) { return __uint_as_float(h & 0x80000000u ? h & 0x7fffffffu : ~h); }

constexpr int TPB = 256, WARPS = TPB / 32, BINS = 2048, CHUNKS = 2048;

// A row's weights: of a logit, in 64 bits and as a whole number.
struct Weights {
  double c, m, unit;
  __device__ double of(float x) const { return exp((double(x) - m) * c); }
  __device__ u64 whole(float x) const { return u64(of(x) * unit + 0.5); }
};

// The largest whole number not above u all, u in [0, 1), exactly.
__device__ __forceinline__ u64 share_of(float u, u64 all) {
  const uint32_t b = __float_as_uint(u);
  const int e = int(b >> 23);        // u = f 2^(max(e, 1) - 150)
  const u64 f = (b & 0x7fffffu) | (e ? 0x800000u : 0u);
  const int down = 150 - (e ? e : 1);          // at least 24
  const u64 lo = f * all, hi = __umul64hi(f, all);
  return down < 64 ? hi << (64 - down) | lo >> down : down < 128 ? hi >> (down - 64) : 0;
}

struct Cut { uint32_t order; int64_t ties, all; };       // kept: larger orders, and the first `ties` of the `all` tokens of this order

struct Smem {
  u64 bin[BINS];
  u64 warp[WARPS];
  u64 found, before;
  int bin_found;
  float max[WARPS];
};

// The sum of v over the threads before this one (after: of all threads in `all`).
__device__ __forceinline__ u64 scan_before(u64 v, Smem& s, u64& all) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  u64 incl = v;
  for (int o = 1; o < 32; o <<= 1) {
    const u64 y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();
  if (lane == 31) s.warp[w] = incl;
  __syncthreads();
  u64 at = incl - v;
  all = 0;
  for (int i = 0; i < WARPS; ++i) {
    at += i < w ? s.warp[i] : 0;
    all += s.warp[i];
  }
  return at;
}

// Cuts the tokens that `floor` keeps (all of them: null) to the shortest start, in descending order, that holds at least `target` (> 0)
// of what `amount` gives to each; there is one.  Three steps over 11, 11 and 10 bits of the order.
template <typename X, typename F>
__device__ Cut cut_row(const X* row, int64_t V, u64 target, const Cut* floor, F&& amount, Smem& s) {
  uint32_t prefix = 0;
  u64 before = 0;
  int shift = 32;
  for (int step = 0; step < 3; ++step) {
    const int bits = step < 2 ? 11 : 10, next = shift - bits;
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += TPB) s.bin[i] = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < V; i += TPB) {
      const float x = to_f(row[i]);
      const uint32_t h = order_of(x);
      if ((shift == 32 || h >> shift == prefix) && (!floor || h >= floor->order)) {
        const u64 v = amount(x);
        if (v) atomicAdd(&s.bin[(h >> next) & ((1u << bits) - 1)], v);
      }
    }
    __syncthreads();
    if (floor && threadIdx.x == 0 && (shift == 32 || floor->order >> shift == prefix))   // the tokens of the floor's own order that it drops
      s.bin[(floor->order >> next) & ((1u << bits) - 1)] -= amount(value_of(floor->order)) * u64(floor->all - floor->ties);
    __syncthreads();
    // bins in descending order, eight per thread
    constexpr int PER = BINS / TPB;
    u64 mine = 0, all;
    for (int j = 0; j < PER; ++j) mine += s.bin[BINS - 1 - (threadIdx.x * PER + j)];
    u64 at = before + scan_before(mine, s, all);
    for (int j = 0; j < PER; ++j) {
      const int b = BINS - 1 - (threadIdx.x * PER + j);
      if (at < target && target <= at + s.bin[b]) {
        s.bin_found = b;
        s.before = at;
      }
      at += s.bin[b];
    }
    __syncthreads();
    prefix = prefix << bits | uint32_t(s.bin_found);
    before = s.before;
    shift = next;
  }
  // the tokens of this order, each with the same amount
  const u64 each = amount(value_of(prefix));
  u64 n = 0, all;
  for (int64_t i = threadIdx.x; i < V; i += TPB) n += order_of(to_f(row[i])) == prefix;
  scan_before(n, s, all);
  Cut c = {prefix, int64_t((target - before + each - 1) / each), int64_t(all)};
  return c;
}

template <typename X>
__global__ void __launch_bounds__(TPB) k_sample(const X* __restrict__ logits, const __grid_constant__ SampleArgs a) {
  __shared__ Smem s;
  __shared__ u64 s_chunk[CHUNKS];
  __shared__ int64_t s_last;
  const int64_t t = blockIdx.x;
  const X* row = logits + t * a.ld;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  auto finish = [&](int64_t token, float logprob) {
    if (a.id_type == MV_I32) static_cast<int32_t*>(a.token)[t] = int32_t(token);
    else static_cast<int64_t*>(a.token)[t] = token;
    if (a.logprob) a.logprob[t] = logprob;
  };
  const float scale = a.scale ? a.scale[t] : 1.0f, u = a.u[t];
  float p = a.top_p ? a.top_p[t] : 1.0f, mp = a.min_p ? a.min_p[t] : 0.0f;
  int64_t k = a.top_k ? a.top_k[t] : 0;
  float m = -INFINITY;
  for (int64_t i = threadIdx.x; i < a.V; i += TPB) m = max_nan(m, to_f(row[i]));
  for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) s.max[w] = m;
  __syncthreads();
  for (int i = 0; i < WARPS; ++i) m = max_nan(m, s.max[i]);
  if (!(m < INFINITY) || !(scale > 0.0f && scale < INFINITY) || isnan(p) || isnan(mp) || isnan(u) || m == -INFINITY) {
    if (threadIdx.x == 0) finish(-1, m == -INFINITY && scale > 0.0f && scale < INFINITY && !isnan(p) && !isnan(mp) && !isnan(u) ? -INFINITY : NAN);
    return;
  }
  if (p <= 0.0f || mp > 1.0f) k = 1;
  mp = fminf(mp, 1.0f);
  if (k <= 0 || k > a.V) k = a.V;
  const Weights wt = {double(scale), double(m), a.unit};
  Cut cut = {0, 0, 0};               // all
  bool cuts = false;
  if (k < a.V) {
    cut = cut_row(row, a.V, u64(k), nullptr, [](float) { return u64(1); }, s);
    cuts = true;
  }
  if (p < 1.0f && p > 0.0f) {
    u64 mine = 0, all;
    for (int64_t i = threadIdx.x; i < a.V; i += TPB) {
      const float x = to_f(row[i]);
      if (!cuts || order_of(x) > cut.order) mine += wt.whole(x);
    }
    scan_before(mine, s, all);
    if (cuts) all += u64(cut.ties) * wt.whole(value_of(cut.order));
    const u64 target = max(u64(1), u64(ceil(double(p) * double(all))));
    cut = cut_row(row, a.V, target, cuts ? &cut : nullptr, [&](float x) { return wt.whole(x); }, s);
    cuts = true;
  }
  // the index of the last kept token of the cut's own order
  int64_t last = a.V;
  if (cuts && cut.ties < cut.all) {
    u64 found = 0;
    for (int64_t i0 = 0; i0 < a.V; i0 += TPB) {
      const int64_t i = i0 + threadIdx.x;
      const bool tie = i < a.V && order_of(to_f(row[i])) == cut.order;
      u64 all;
      const u64 at = found + scan_before(tie, s, all);
      if (tie && at + 1 == u64(cut.ties)) s_last = i;
      found += all;
      if (found >= u64(cut.ties)) break;
    }
    __syncthreads();
    last = s_last;
  }
  auto kept = [&](int64_t i) {       // the weight of token i, 0 if it is cut
    const float x = to_f(row[i]);
    const uint32_t h = order_of(x);
    if (cuts && !(h > cut.order || (h == cut.order && i <= last))) return u64(0);
    const double v = wt.of(x);
    return v >= double(mp) ? u64(v * wt.unit + 0.5) : u64(0);
  };
  const int64_t per = ((a.V + CHUNKS - 1) / CHUNKS + 31) / 32 * 32;
  __syncthreads();
  for (int c = w; c < CHUNKS; c += WARPS) {
    u64 n = 0;
    for (int64_t i = c * per + lane; i < min(a.V, (c + 1) * per); i += 32) n += kept(i);
    for (int o = 16; o; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    if (lane == 0) s_chunk[c] = n;
  }
  __syncthreads();
  constexpr int PER = CHUNKS / TPB;
  u64 mine = 0, all;
  for (int j = 0; j < PER; ++j) mine += s_chunk[threadIdx.x * PER + j];
  u64 at = scan_before(mine, s, all);
  const u64 limit = u >= 1.0f ? all - 1 : u > 0.0f ? share_of(u, all) : 0;       // the first token at which the sum is larger is drawn
  for (int j = 0; j < PER; ++j) {
    const u64 n = s_chunk[threadIdx.x * PER + j];
    if (at <= limit && limit < at + n) {
      s.bin_found = threadIdx.x * PER + j;
      s.before = at;
    }
    at += n;
  }
  __syncthreads();
  if (w) return;
  u64 before = s.before;
  for (int64_t i0 = s.bin_found * per; i0 < a.V; i0 += 32) {
    const int64_t i = i0 + lane;
    const u64 n = i < a.V ? kept(i) : 0;
    u64 incl = n;
    for (int o = 1; o < 32; o <<= 1) {
      const u64 y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, before + incl > limit);
    if (hit) {
      if (lane == __ffs(int(hit)) - 1) finish(i, float((double(to_f(row[i])) - wt.m) * wt.c - log(double(all) / wt.unit)));
      return;
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
}

}  // namespace

extern "C" {

int mv_sample(void* stream, const void* logits, int type, int64_t T, int64_t V, int64_t ld, const float* u, const float* scale,
              const int32_t* top_k, const float* top_p, const float* min_p, void* token, int id_type, float* logprob) {
  const int64_t lim = int64_t(1) << 31;
  if (!is_value_type(type) || T < 0 || T >= lim || V < 1 || V >= lim || ld < V || (T > 0 && (!logits || !u || !token)) || misaligned(logits, type_size(type)) ||
      !is_id_type(id_type) || misaligned(token, type_size(id_type)) || misaligned(u, 4) || misaligned(scale, 4) || misaligned(top_k, 4) || misaligned(top_p, 4) ||
      misaligned(min_p, 4) || misaligned(logprob, 4))
    return MV_ERR_INVALID_ARG;
  if (T == 0) return MV_OK;
  SampleArgs a;
  a.V = V; a.ld = ld; a.unit = ldexp(1.0, 61); a.u = u;
  for (int64_t n = 1; n < V; n *= 2) a.unit *= 0.5; a.scale = scale; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.token = token; a.id_type = id_type; a.logprob = logprob;
  return with_type(type, [&](auto x) {
    using X = decltype(x);
    k_sample<X><<<unsigned(T), TPB, 0, static_cast<cudaStream_t>(stream)>>>(static_cast<const X*>(logits), a);
    return cuda_ok();
  });
}

}  // extern "C"
