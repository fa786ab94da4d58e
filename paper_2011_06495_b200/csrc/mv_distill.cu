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

// A row's alternatives in shared memory: columns (-1: none), log probabilities (-inf there), and one more number each.
struct List {
  int* col;
  float *a, *x;
  __device__ __forceinline__ List(void* smem, int k) : col(static_cast<int*>(smem)), a(reinterpret_cast<float*>(col + k)), x(a + k) {}
};
constexpr int LIST_BYTES = 12;

// want(column): whether its logit is asked for.
template <typename X, typename F> __device__ __forceinline__ void load_list(const Teacher& h, int64_t t, int64_t V, const X* row, const List& s, F&& want) {
  for (int j = threadIdx.x; j < h.k; j += blockDim.x) {
    const int c = int(load_id(h.id, h.id_type, t * h.k + j, V));
    s.col[j] = c;
    s.a[j] = c < 0 ? -INFINITY : h.top[t * h.k + j];
    s.x[j] = c >= 0 && want(c) ? to_f(row[c]) : -INFINITY;
  }
}

struct DistillArgs {
  int64_t V, ld;
  Teacher h;
  float scale;
  int marks;                         // words of marks that a row needs, at most MARKS
  float *kl, *lse, *log_rest;
};

constexpr int U = 4;                 // vectors per thread and step, all in flight, two by two from neighbouring places
constexpr int MARKS = 4096;          // words of marks: one for each thread and step, a bit for each of its logits

// A CTA per row, streamed once with a running reference.  With the rest as a class the listed tokens are kept out of the sum (taking them
// off it would leave nothing of a small rest): a bit for every logit of the next steps, set for the listed ones, which a thread asks
// one word at a time; their own terms are added at the end.  Memory bounds it: 8192 x 65536 bf16 with 32 alternatives 173 us (6.2 TB/s), with
// the rest 183 (5.9).  The end of a row, some microseconds of latency for its list, is covered by the other CTAs unless rows are short
// (16000 x 8000 68 us, floor 39; 16384 x 1000 f16 with 50 alternatives 50, floor 6) or few (64 x 131072: 19 us, floor 2.6: a CTA a row).  Times
// here and below are those of calls that follow one another for half a second, at the power limit; in short runs those that memory
// bounds take up to a tenth less (161 and 169 us), and the two sides of a rule were compared like that.
// (Its sums are in 32 bits: lse, log P and so each log p are; the list's sums and the divergence in 64.)
template <typename X, bool REST, int TPB>
__global__ void __launch_bounds__(TPB, 1024 / TPB) k_distill(const X* __restrict__ logits, const __grid_constant__ DistillArgs a) {
  constexpr int N = Vec<X>::N, WARPS = TPB / 32, WINDOW = MARKS / TPB;
  extern __shared__ uint32_t dynamic[];
  __shared__ float s_max[WARPS], s_ref[WARPS], s_sum[WARPS];
  __shared__ uint32_t s_ends;
  __shared__ int s_twice;
  uint32_t* mark = dynamic;          // [step of the window][thread], with REST
  const List list(dynamic + (REST ? a.marks : 0), a.h.k);
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const X* row = logits + t * a.ld;
  // the vectors begin at the row's first 32-byte boundary
  const int64_t to32 = int64_t((32 - (reinterpret_cast<uintptr_t>(row) & 31)) & 31) / int(sizeof(X));
  const int first = int(min(a.V, to32)), nv = (int(a.V) - first) / (2 * N) * 2, tail_col = first + nv * N, ends = first + int(a.V) - tail_col;
  const uint4* vec = reinterpret_cast<const uint4*>(row + first);
  const uint4 none = make_uint4(Vec<X>::NONE, Vec<X>::NONE, Vec<X>::NONE, Vec<X>::NONE);
  const int n_full = nv / (TPB * U), n_steps = (nv + TPB * U - 1) / (TPB * U);
  auto load = [&](int step, uint4 (&u)[U]) {
    const uint4* ptr = vec + step * (U * TPB) + 2 * tid;
    if (step < n_full) {
#pragma unroll
      for (int i = 0; i < U; i += 2) load_stream(ptr + i * TPB, u[i], u[i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < U; i += 2) {
        u[i] = u[i + 1] = none;
        if ((step * U + i) * TPB + 2 * tid < nv) load_stream(ptr + i * TPB, u[i], u[i + 1]);
      }
    }
  };
  uint4 even[U], odd[U];
  if (n_steps > 0) load(0, even);
  if (tid == 0) { s_ends = 0; s_twice = 0; }
  load_list(a.h, t, a.V, row, list, [](int) { return true; });
  // marks the listed tokens of the steps [step, step + WINDOW); the ends with the first ones
  auto set_marks = [&](int step) {
    __syncthreads();                 // the marks before have been read
    for (int i = tid; i < min(MARKS, (n_steps - step) * TPB); i += TPB) mark[i] = 0;
    __syncthreads();
    for (int j = tid; j < a.h.k; j += TPB) {
      const int c = list.col[j];
      uint32_t bit, old = 0;
      if (c < 0) continue;
      if (c < first || c >= tail_col) {
        bit = 1u << (c < first ? c : first + c - tail_col);
        if (step == 0) old = atomicOr(&s_ends, bit);
      } else {
        const unsigned v = unsigned(c - first) / N, s = v / (U * TPB), at = v % (U * TPB), in = at % (2 * TPB);
        bit = 1u << ((at / (2 * TPB) * 2 + (in & 1)) * N + unsigned(c - first) % N);
        if (int(s) >= step && int(s) < step + WINDOW) old = atomicOr(mark + (s - step) * TPB + in / 2, bit);
      }
      if (old & bit) s_twice = 1;
    }
    __syncthreads();
  };
  if constexpr (REST) set_marks(0);
  const bool my_end = tid < ends, end_listed = REST && my_end && (s_ends >> tid & 1u);
  const float end = my_end ? to_f(row[tid < first ? tid : tail_col + tid - first]) : -INFINITY;
  const float c2 = fminf(a.scale * LOG2E, 3.0e38f), room = LAG / c2;
  const f2 c22 = pack2(c2, c2);
  // logits below the first limit never set the reference; beside a reference above -R_MAX their 2^t is 0
  float ref = -INFINITY, R = 0.0f, limit = -2.0f * R_MAX / c2, largest = end;
  f2 minus = pack2(0.0f, 0.0f), s2 = pack2(0.0f, 0.0f);
  auto raise = [&](float m) {        // a new reference
    const float Rm = m * c2;
    if (ref != -INFINITY) {
      float p0, p1;
      unpack2(s2, p0, p1);
      s2 = pack2((p0 + p1) * exp2_fast(max_nan(R - Rm, T_FLOOR)), 0.0f);
    }
    ref = m;
    R = Rm;
    limit = m + room;
    minus = pack2(-Rm, -Rm);
  };
  auto add_pair = [&](f2 v) {
    float u0, u1;
    unpack2(fma2(v, c22, minus), u0, u1);
    s2 = add2(s2, pack2(exp2_fast(u0), exp2_fast(u1)));
  };
  auto hide = [&](int step, uint4 (&u)[U]) {          // the listed logits of a step become masked ones
    const uint32_t word = mark[step % WINDOW * TPB + tid];
    if (word == 0) return;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      uint32_t q[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (word >> (i * N + e) & 1u) {
          if constexpr (N == 4) q[e] = Vec<X>::NONE;
          else q[e / 2] = e % 2 ? (q[e / 2] & 0xffffu) | (Vec<X>::NONE & 0xffff0000u) : (q[e / 2] & 0xffff0000u) | (Vec<X>::NONE & 0xffffu);
        }
      u[i] = make_uint4(q[0], q[1], q[2], q[3]);
    }
  };
  auto take = [&](int step, uint4 (&u)[U]) {
    uint32_t m2 = Vec<X>::max2(Vec<X>::max2(u[0].x, u[0].y), Vec<X>::max2(u[0].z, u[0].w));
#pragma unroll
    for (int i = 1; i < U; ++i) m2 = Vec<X>::max2(m2, Vec<X>::max2(Vec<X>::max2(u[i].x, u[i].y), Vec<X>::max2(u[i].z, u[i].w)));
    const float m = Vec<X>::widen(m2);
    if (m > limit) raise(m);
    largest = fmaxf(largest, m);
    if constexpr (REST) hide(step, u);
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int j = 0; j < N / 2; ++j) add_pair(Vec<X>::pair(u[i], j));
  };
  if (my_end) {
    if (end > limit) raise(end);
    add_pair(pack2(end_listed ? -INFINITY : end, -INFINITY));
  }
  for (int step = 0; step < n_steps; step += 2) {
    if (step + 1 < n_steps) load(step + 1, odd);
    if (REST && step && step % WINDOW == 0) set_marks(step);
    take(step, even);
    if (step + 1 >= n_steps) break;
    if (step + 2 < n_steps) load(step + 2, even);
    take(step + 1, odd);
  }
  float sum;
  {
    float p0, p1;
    unpack2(s2, p0, p1);
    const float d = ref == -INFINITY ? 0.0f : fmaf(ref, c2, -R);      // at most half a unit of R; 2^-d
    sum = (p0 + p1) * fmaf(fmaf(0.5f * LN2 * LN2, d, -LN2), d, 1.0f);
  }
  // the largest logit, and the sums relative to it
  for (int o = 16; o; o >>= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, o));
  if (lane == 0) s_max[w] = largest;
  __syncthreads();
  for (int i = 0; i < WARPS; ++i) largest = fmaxf(largest, s_max[i]);
  const float top = largest, zero = top == -INFINITY ? 0.0f : top;
  if (top * c2 > R_MAX || c2 < C2_MIN || (top * c2 < -R_MAX && top > -INFINITY)) {
    // logits that the fused form cannot take: summed again by differences to the largest one
    sum = 0.0f;
    auto add = [&](float v) { sum += exp2_fast(distance(v, zero, c2)); };
    if (my_end && !end_listed) add(end);
    for (int step = 0; step < n_steps; ++step) {
      if (REST && step % WINDOW == 0) set_marks(step);
      load(step, even);
      if constexpr (REST) hide(step, even);
#pragma unroll
      for (int i = 0; i < U; ++i) each_logit<X>(even[i], [&](int, float v) { add(v); });
    }
  } else if (ref != top) {
    sum = ref == -INFINITY ? sum : sum * exp2_fast(max_nan(distance(ref, zero, c2), T_FLOOR));
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[w] = sum;
  __syncthreads();
  if (w) return;
  sum = 0.0f;
  for (int i = 0; i < WARPS; ++i) sum += s_sum[i];
  // the listed tokens' own terms, each token once
  double all = sum, own = 0.0;
  if constexpr (REST) {
    for (int j = lane; j < a.h.k; j += 32) {
      const int c = list.col[j];
      bool again = c < 0;
      if (s_twice)
        for (int i = 0; i < j && !again; ++i) again = list.col[i] == c;
      if (!again) own += double(exp2_fast(distance(list.x[j], zero, c2)));
    }
    for (int o = 16; o; o >>= 1) own += __shfl_xor_sync(0xffffffffu, own, o);
    all += own;
  }
  // With e_j = exp(a_j - shift): q_j = e_j / sum e without the rest (shift: the largest a_j), e_j with it (shift 0).  1 - sum q is a small
  // difference, so these are in 64 bits.
  // log P by what is missing to one where that is the smaller part: the difference of two logarithms would lose it.
  const float ls = logf(float(all)), lr = own > 0.0 && own < sum ? log1pf(-float(own / all)) : logf(sum) - ls;
  float m = -INFINITY;
  bool any = false, bad = false;
  for (int j = lane; j < a.h.k; j += 32) {
    const float v = list.a[j];
    any |= list.col[j] >= 0 && (REST || v != -INFINITY);
    bad |= !(v < INFINITY);
    m = fmaxf(m, v);
  }
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  any = __any_sync(0xffffffffu, any);
  bad = __any_sync(0xffffffffu, bad);
  const double shift = REST || m == -INFINITY ? 0.0 : double(m);
  double q = 0.0, kl = 0.0;
  for (int j = lane; j < a.h.k; j += 32) {
    const double d = double(list.a[j]) - shift, e = exp(d);
    q += e;
    if (e > 0.0) kl = fma(e, d - ((double(list.x[j]) - double(zero)) * double(a.scale) - double(ls)), kl);      // (in 32 bits a finite mask may pass the range)
  }
  for (int o = 16; o; o >>= 1) {
    q += __shfl_xor_sync(0xffffffffu, q, o);
    kl += __shfl_xor_sync(0xffffffffu, kl, o);
  }
  if (lane == 0) {
    const bool nan = isnan(all), empty = all == 0.0;
    if (!REST) {
      kl = kl / q - log(q);
    } else if (any && q < 1.0) {
      const double rest = 1.0 - q;
      kl += rest * (log(rest) - double(lr));
    }
    if (a.kl) a.kl[t] = !any ? 0.0f : nan || bad ? NAN : empty ? INFINITY : float(kl);
    if (a.lse) a.lse[t] = nan ? NAN : empty ? -INFINITY : fmaf(a.scale, zero, ls);
    if (a.log_rest) a.log_rest[t] = nan ? NAN : empty ? -INFINITY : lr;
  }
}

// ------------------------------------------------------------------------------------------ gradient
// dx = f (M p - q) for a listed token, f M' p for the others, f = c g, M' = M - r / P.  p = q q with q = 2^h, h = log2(p) / 2: the
// hardware's exponential has no subnormal results.  Each CTA takes some stretches of one row, and all of the row's list: the others' value is
// written everywhere, and then its listed tokens' over it.  Memory bounds it: 8192 x 65536 bf16 354 us (6.1 TB/s in and out), 4096 x
// 131072 with 64 alternatives 353; 9000 x 33001 f16 196 us, with rows that lie differently within 16 bytes 219 (element by element 877).
// Short rows wait for their lists: 16384 x 1000 f16 with 50 alternatives 47 us (floor 11); so do long lists, all of which every CTA works out:
// 2000 x 151936 bf16 with 1024 alternatives 364 us (floor 188).  The shares e_j are kept in 32 bits, half a unit of a result of 32 bits.
constexpr int GRAD_U = 4, GRAD_EACH = 4;

struct DistillGradArgs {
  int64_t V, ld, ldg;
  Teacher h;
  float scale;
  unsigned ctas;                     // per row
  int stretches;                     // per CTA
  const float *lse, *log_rest, *g;
};

// APART: logits and gradient do not start at the same place within 16 bytes in every row; then the vectors are the gradient's, and the logits
// come from between two of theirs.
template <typename X, bool APART, int TPB>
__global__ void __launch_bounds__(TPB) k_distill_grad(const X* logits, X* dlogits, const __grid_constant__ DistillGradArgs a) {
  constexpr int N = Vec<X>::N, WARPS = TPB / 32, SEEN = 128;
  extern __shared__ uint32_t dynamic[];
  __shared__ float s_max[WARPS];
  __shared__ double s_sum[WARPS];
  __shared__ uint32_t s_seen[2][SEEN];
  const List list(dynamic, a.h.k);
  const int64_t t = blockIdx.x / a.ctas;
  const unsigned part = blockIdx.x % a.ctas;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const X* x = logits + t * a.ld;
  X* dx = dlogits + t * a.ldg;
  // the vectors begin at a 16-byte boundary of the gradient's row; what is before and behind them goes to the first stretch
  int64_t first = min(a.V, int64_t((16 - (reinterpret_cast<uintptr_t>(dx) & 15)) & 15) / int(sizeof(X)));
  const int shift = APART ? int(reinterpret_cast<uintptr_t>(x + first) & 15) : 0;       // where in a vector of the logits
  if (shift > first * int(sizeof(X))) first = min(a.V, first + N);                       // all of the two vectors' bytes are the row's
  const int64_t nv = max(int64_t(0), (a.V - first - (APART ? N - shift / int(sizeof(X)) : 0)) / N), behind = first + nv * N, ends = first + a.V - behind;
  const int64_t v0 = int64_t(part) * a.stretches * (TPB * GRAD_U), v1 = min(nv, v0 + a.stretches * (TPB * GRAD_U));      // its vectors
  const int64_t c0 = first + v0 * N, c1 = min(behind, c0 + a.stretches * (TPB * GRAD_U * N));                                            // and columns
  const uint4* in = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(x + first) - shift);
  uint4* out = reinterpret_cast<uint4*>(dx + first);
  const bool my_end = part == 0 && tid < ends;
  const int64_t end_col = tid < first ? tid : behind + tid - first;
  uint4 u[GRAD_U], next[GRAD_U], more[APART ? GRAD_U : 1];
  auto load = [&](int64_t v) {
#pragma unroll
    for (int i = 0; i < GRAD_U; ++i)
      if (v + i * TPB < v1) {
        if constexpr (APART) {
          next[i] = __ldg(in + v + i * TPB);
          more[i] = __ldg(in + v + i * TPB + 1);
        } else {
          next[i] = __ldcs(in + v + i * TPB);
        }
      }
  };
  load(v0 + tid);
  const float end = my_end ? to_f(x[end_col]) : 0.0f;
  auto here = [&](int64_t c) { return (c >= c0 && c < c1) || (part == 0 && c >= 0 && (c < first || c >= behind)); };      // the CTA's columns
  for (int i = tid; i < 2 * SEEN; i += TPB) s_seen[i / SEEN][i % SEEN] = 0;
  load_list(a.h, t, a.V, x, list, here);
  const float l = a.lse[t], g = a.g[t], lr = a.h.rest ? a.log_rest[t] : 0.0f;
  // e_j as in the forward pass, in the place of a_j; their sum in 64 bits
  float m = -INFINITY;
  bool any = false, bad = false;
  for (int j = tid; j < a.h.k; j += TPB) {
    const float v = list.a[j];
    any |= list.col[j] >= 0 && (a.h.rest || v != -INFINITY);
    bad |= !(v < INFINITY);
    m = fmaxf(m, v);
  }
  any = __syncthreads_or(any);
  bad = __syncthreads_or(bad);
  if (!a.h.rest) {
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) s_max[w] = m;
    __syncthreads();
    for (int i = 0; i < WARPS; ++i) m = fmaxf(m, s_max[i]);
  }
  const double base = a.h.rest || m == -INFINITY ? 0.0 : double(m);
  double sum = 0.0;
  for (int j = tid; j < a.h.k; j += TPB) {
    const double e = exp(double(list.a[j]) - base);
    sum += e;
    list.a[j] = float(e);
    const int c = list.col[j];
    if (here(c)) {                   // its place among SEEN * 32: taken once, or more than once
      const uint32_t bit = 1u << (c & 31);
      if (atomicOr(&s_seen[0][c / 32 % SEEN], bit) & bit) atomicOr(&s_seen[1][c / 32 % SEEN], bit);
    }
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[w] = sum;
  __syncthreads();
  sum = 0.0;
  for (int i = 0; i < WARPS; ++i) sum += s_sum[i];
  const double r = a.h.rest ? fmax(0.0, 1.0 - sum) : 0.0;
  const float all = bad ? NAN : a.h.rest ? float(sum + r) : 1.0f;
  const double unit = a.h.rest ? 1.0 : 1.0 / sum;
  const float ratio = r == 0.0 ? 0.0f : lr == -INFINITY ? all : expf(logf(float(r)) - lr);
  const bool none = !any || g == 0.0f || l == -INFINITY || a.scale * g == 0.0f;
  // r / P may pass the range of 32 bits where P is small; p_v r / P does not.  Then the others are f (p_v / P) (M P - r).
  const bool far = r > 0.0 && lr > -INFINITY && lr < -40.0f;
  const float f = none ? 0.0f : a.scale * g, other = f * (far ? all * expf(lr) - float(r) : all - ratio), l2e = 0.5f * LOG2E;
  const float lo = far ? l + lr : l, most = far ? -lr * l2e : 0.0f;            // of p_v / P, or of p_v: its log, and at most how much (p_v: 1)
  auto share = [&](float v, float base, float most) {       // p / q, or p / P / q; the same operations as two logits at a time below
    return exp2_fast(min_nan(fmaf(v, a.scale, -base) * l2e, most));
  };
  auto one = [&](float v) {
    const float q = share(v, lo, most);
    return none ? 0.0f : q * (q * other);
  };
  const f2 scale2 = pack2(a.scale, a.scale), minus = pack2(-lo, -lo), l2e2 = pack2(l2e, l2e), other2 = pack2(other, other);
  for (int64_t vs = v0 + tid; vs < v1; vs += TPB * GRAD_U) {
#pragma unroll
    for (int i = 0; i < GRAD_U; ++i) {
      if constexpr (APART) u[i] = between(next[i], more[i], shift);
      else u[i] = next[i];
    }
    load(vs + TPB * GRAD_U);
#pragma unroll
    for (int i = 0; i < GRAD_U; ++i) {
      const int64_t v = vs + i * TPB;
      if (v >= v1) break;
      float d[N];
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        float h0, h1;
        unpack2(mul2(fma2(Vec<X>::pair(u[i], j), scale2, minus), l2e2), h0, h1);
        const f2 q = pack2(exp2_fast(min_nan(h0, most)), exp2_fast(min_nan(h1, most)));
        unpack2(mul2(q, mul2(q, other2)), d[2 * j], d[2 * j + 1]);
      }
      __stcs(out + v, none ? make_uint4(0, 0, 0, 0) : pack_vec<X>(d));
    }
  }
  if (my_end) dx[end_col] = from_f<X>(one(end));
  if (none) return;
  // the CTA's listed tokens, each by the thread of its first entry
  bool mine = false;
  for (int j = tid; j < a.h.k; j += TPB) mine |= here(list.col[j]);
  if (!__syncthreads_or(mine)) return;
  for (int j = tid; j < a.h.k; j += TPB) {
    const int c = list.col[j];
    if (!here(c)) continue;
    double q = list.a[j];            // (its terms are of 32 bits, their sum is not: a token may have all k of them)
    bool head = true;
    if (s_seen[1][c / 32 % SEEN] >> (c & 31) & 1u) {
      q = 0.0;
      for (int i = 0; i < a.h.k; ++i)
        if (list.col[i] == c) {
          head &= i >= j;
          q += double(list.a[i]);
        }
    }
    const float p = share(list.x[j], l, 0.0f);
    if (head) dx[c] = from_f<X>(f * fmaf(all * p, p, -float(q * unit)));
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
  // a row's results are written while other rows are read
  for (const float* p : {kl, lse, log_rest})
    if (share_vector(p, T, 4, logits, T, V, ld, type_size(type)) || share_vector(p, T, 4, top_logprob, T, k, k, 4) ||
        share_vector(p, T, 4, top_id, T, k, k, type_size(id_type)))
      return MV_ERR_INVALID_ARG;
  if (share_vector(kl, T, 4, lse, 1, T, T, 4) || share_vector(kl, T, 4, log_rest, 1, T, T, 4) || share_vector(lse, T, 4, log_rest, 1, T, T, 4))
    return MV_ERR_INVALID_ARG;
  DistillArgs a;
  a.V = V; a.ld = ld; a.h = {top_logprob, top_id, id_type, k, rest}; a.scale = scale; a.kl = kl; a.lse = lse; a.log_rest = log_rest;
  return with_type(type, [&](auto x) {
    using X = decltype(x);
    const int64_t vecs = V / Vec<X>::N;
    // short rows take few threads and many CTAs, if there are rows enough to fill the device; long or few rows many threads (the sides of
    // this rule as measured for the log probabilities, whose stream is the same)
    const int tpb = T >= 1184 && vecs <= 3000 ? 64 : vecs > 10240 || (T < 600 && vecs > 6000) ? 256 : 128;
    const int64_t words = (vecs + tpb * U - 1) / (tpb * U) * tpb;
    a.marks = !rest ? 0 : words > MARKS ? MARKS : int(words);        // short rows leave room for more CTAs
    const size_t smem = size_t(k) * LIST_BYTES + size_t(a.marks) * 4;
    auto launch = [&](auto r) {
      constexpr bool REST = decltype(r)::value;
      auto* kernel = tpb == 64 ? k_distill<X, REST, 64> : tpb == 128 ? k_distill<X, REST, 128> : k_distill<X, REST, 256>;
      kernel<<<unsigned(T), unsigned(tpb), smem, static_cast<cudaStream_t>(stream)>>>(static_cast<const X*>(logits), a);
      return cuda_ok();
    };
    return rest ? launch(std::true_type()) : launch(std::false_type());
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
  for (const float* p : {lse, log_rest, g})            // which a row's other CTAs may have yet to read
    if (share_vector(p, T, 4, dlogits, T, V, ldg, size)) return MV_ERR_INVALID_ARG;
  DistillGradArgs a;
  a.V = V; a.ld = ld; a.ldg = ldg; a.h = {top_logprob, top_id, id_type, k, log_rest ? 1 : 0}; a.scale = scale; a.lse = lse; a.log_rest = log_rest; a.g = g;
  return with_type(type, [&](auto x) {
    using X = decltype(x);
    // The list costs a CTA a few microseconds of latency: as many stretches for each as leave enough CTAs to fill the device, up to a CTA for
    // four, or for a few more than to leave a row's last CTA with fewer (4096 x 131072 bf16 with 64 alternatives, 16 stretches: one each
    // 476 us, two 383, four 338, eight 346, sixteen 361; 9000 x 33001, five: four and one 219, together 194).  Where the device's fill
    // decides, a row's last CTA has what is left (five as four and one from 948 to 1183 rows: 1003 x 33001 31 us).  Rows of up to 16 KB
    // take small CTAs (16000 x 8000 bf16: 90 us, with 256 threads 138).
    const int tpb = V * size <= 16384 ? 64 : 256;
    const int64_t per = int64_t(tpb) * GRAD_U * Vec<X>::N, stretches = (V + per - 1) / per;
    const int64_t least = stretches < 2 * GRAD_EACH ? 1 : stretches / GRAD_EACH, most = (stretches + least - 1) / least;
    int64_t each = T * stretches / (148 * 2048 / tpb);
    each = each < 1 ? 1 : each > most ? most : each;
    a.stretches = int(each);
    a.ctas = unsigned((stretches + each - 1) / each);
    if (T * a.ctas >= lim) return int(MV_ERR_INVALID_ARG);
    const bool vec = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(dlogits)) & 15) == 0 && (T == 1 || (ld - ldg) * int64_t(sizeof(X)) % 16 == 0);
    auto* kernel = tpb == 64 ? (vec ? k_distill_grad<X, false, 64> : k_distill_grad<X, true, 64>) : vec ? k_distill_grad<X, false, 256> : k_distill_grad<X, true, 256>;
    kernel<<<unsigned(T * a.ctas), unsigned(tpb), size_t(k) * LIST_BYTES, static_cast<cudaStream_t>(stream)>>>(static_cast<const X*>(logits), static_cast<X*>(dlogits), a);
    return cuda_ok();
  });
}

}  // extern "C"
