// mv_token.cu -- log probabilities of given tokens with entropy and alternatives, and their gradient, for sm_100a.
//
// With z = c x, r a reference near the row's largest logit and t = (x - r) c log2(e):  s = sum 2^t,  lse = c r + log s,
// H = log s - ln 2 (sum 2^t t) / s.  A masked logit (-inf) has 2^t = 0 and must not multiply its t, so t is kept above a
// finite floor.  t is one fused multiply-add, x (c log2 e) - R with R = r c log2(e) rounded; what the rounding of R costs is put
// right once per thread.  Rows in which R itself would overflow (every logit near the type's lowest or largest value) are
// summed again in a form that takes the difference first.

#include "mv_lm.cuh"

#include <cooperative_groups.h>
#include <math.h>

namespace {

namespace cg = cooperative_groups;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float T_FLOOR = -1.0e30f;
constexpr float R_MAX = 1.0e37f;     // references up to here are summed by the fused form

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
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

__device__ __forceinline__ uint4 load_stream(const uint4* p) {
  uint4 u;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
  return u;
}

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

// One row, or one CTA's part of it: `head` single logits, nv vectors of 16 bytes, `tail` single logits.
template <typename X> struct Part {
  const X* row;
  const uint4* vec;                  // the part's first vector
  int64_t nv;
  uint32_t col0;                     // its column
  uint32_t head, tail, tail_col;
};

// ------------------------------------------------------------------------------------------ alternatives
// The k largest logits cost the streaming pass almost nothing: a thread keeps the largest logit of every group (a few
// vectors) that it reads.  Afterwards a bound B is found that at least k group maxima reach; every logit above B lies in a
// group whose maximum is above B, and those few groups are read again.
constexpr int U = 4;                 // vectors per thread and step, all in flight
constexpr int MAX_GROUPS = 32;       // groups per thread
constexpr int GROUP_LIST = 256;      // groups read again
constexpr int KEY_LIST = 1024;       // candidates

struct TopSmem {
  unsigned long long key[KEY_LIST];
  unsigned long long best[MV_TOP_MAX];
  uint16_t group[GROUP_LIST];
  float sorted[16][32];              // of each warp
  float bound;
  int n_key, n_group, n_above, found;
};

// Sorts a warp's 32 values in descending order.
__device__ __forceinline__ float sort_warp(float v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j; j >>= 1) {
      const float o = __shfl_xor_sync(0xffffffffu, v, j);
      const bool up = ((lane & k) == 0) == ((lane & j) == 0);         // this lane keeps the larger one
      v = up ? fmaxf(v, o) : fminf(v, o);
    }
  return v;
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

// The k best keys of this part, in order, in s.best (0 where there are fewer).  All threads; ends with a barrier.
template <typename X, int TPB>
__device__ void best_of_part(const Part<X>& p, int k, const float* gmax, int groups, int steps, float mine, TopSmem& s) {
  constexpr int WARPS = TPB / 32;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const float sorted = sort_warp(mine);
  s.sorted[w][lane] = sorted;
  if (threadIdx.x == 0) { s.n_key = 0; s.n_group = 0; s.n_above = 0; s.found = 0; }
  if (threadIdx.x < MV_TOP_MAX) s.best[threadIdx.x] = 0;
  __syncthreads();
  if (w == 0) {
    // If j warps hold r maxima >= b each, j r >= k of them reach b: lane r - 1 tries r, with the ceil(k / r)-th largest of the warps' r-th maxima.
    float v[WARPS];
#pragma unroll
    for (int i = 0; i < WARPS; ++i) v[i] = s.sorted[i][lane];
    const int j = (k + lane) / (lane + 1);
    float b = -INFINITY;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
      int reach = 0;
#pragma unroll
      for (int m = 0; m < WARPS; ++m) reach += v[m] >= v[i];
      if (reach >= j) b = fmaxf(b, v[i]);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) b = fmaxf(b, __shfl_xor_sync(0xffffffffu, b, o));
    if (lane == 0) s.bound = b;
  }
  __syncthreads();
  const float B = s.bound;
  auto push = [&](float x, uint32_t col) {
    const int i = atomicAdd(&s.n_key, 1);
    if (i < KEY_LIST) s.key[i] = make_key(x, col);
  };
  if (mine >= B)
    for (int g = 0; g < groups; ++g) {
      const float m = gmax[g * TPB + threadIdx.x];
      if (m > B) atomicAdd(&s.n_above, 1);
      if (m >= B) {
        const int i = atomicAdd(&s.n_group, 1);
        if (i < GROUP_LIST) s.group[i] = uint16_t(g * TPB + threadIdx.x);
      }
    }
  // the single logits at the ends are always candidates
  if (threadIdx.x < p.head + p.tail) {
    const uint32_t col = threadIdx.x < p.head ? threadIdx.x : p.tail_col + threadIdx.x - p.head;
    const float x = to_f(p.row[col]);
    if (x == x) push(x, col);
  }
  __syncthreads();
  const bool few = s.n_group <= GROUP_LIST;
  const int per = steps * U;         // vectors per group
  if (!few && s.n_above > 0) {       // many groups at the bound itself: list the ones above it
    __syncthreads();
    if (threadIdx.x == 0) s.n_group = 0;
    __syncthreads();
    if (mine > B)
      for (int g = 0; g < groups; ++g)
        if (gmax[g * TPB + threadIdx.x] > B) {
          const int i = atomicAdd(&s.n_group, 1);
          if (i < GROUP_LIST) s.group[i] = uint16_t(g * TPB + threadIdx.x);
        }
    __syncthreads();
  }
  const int listed = few || s.n_above > 0 ? min(s.n_group, GROUP_LIST) : 0;
  for (int i = threadIdx.x; i < listed * per; i += TPB) {
    const int gi = s.group[i / per], g = gi / TPB;
    const int64_t v = int64_t(gi % TPB) + (int64_t(g) * per + i % per) * TPB;
    if (v >= p.nv) continue;
    const uint4 u = __ldg(p.vec + v);
    const uint32_t col = p.col0 + uint32_t(v) * Vec<X>::N;
    each_logit<X>(u, [&](int e, float x) {
      if (few ? x >= B : x > B) push(x, col + e);
    });
  }
  __syncthreads();
  bool whole = s.n_above <= GROUP_LIST && s.n_key <= KEY_LIST;
  if (whole && !few) {
    // the logits at the bound, in order from the start of the part until k of them are found (they are many)
    for (int64_t v0 = 0; v0 < p.nv; v0 += TPB) {
      const int64_t v = v0 + threadIdx.x;
      unsigned hit = 0;
      if (v < p.nv) {
        const uint4 u = __ldg(p.vec + v);
        each_logit<X>(u, [&](int e, float x) { hit |= x == B ? 1u << e : 0u; });
      }
      int c = __popc(hit), incl = c;
      for (int o = 1; o < 32; o <<= 1) {
        const int z = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += z;
      }
      if (lane == 31) s.sorted[w][0] = __int_as_float(incl);
      __syncthreads();
      int at = s.found + incl - c, all = s.found;
      for (int i = 0; i < WARPS; ++i) {
        const int n = __float_as_int(s.sorted[i][0]);
        at += i < w ? n : 0;
        all += n;
      }
      for (int e = 0; e < Vec<X>::N; ++e)
        if ((hit >> e & 1u) && at++ < k) push(B, p.col0 + uint32_t(v) * Vec<X>::N + e);
      __syncthreads();
      if (threadIdx.x == 0) s.found = all;
      __syncthreads();
      if (all >= k) break;
    }
    whole = s.n_key <= KEY_LIST;
  }
  if (whole) {
    // every candidate's place is the number of candidates before it
    const int n = s.n_key;
    for (int i = threadIdx.x; i < n; i += TPB) {
      const unsigned long long mykey = s.key[i];
      int place = 0;
      for (int j = 0; j < n; ++j) place += s.key[j] > mykey;
      if (place < k) s.best[place] = mykey;
    }
  } else {
    // too many candidates (large logits crowded in few threads' columns): one reading of the part per alternative
    unsigned long long last = ~0ull;
    for (int r = 0; r < k; ++r) {
      unsigned long long b = 0;
      auto take = [&](float x, uint32_t col) {
        const unsigned long long y = x == x ? make_key(x, col) : 0;
        if (y < last && y > b) b = y;
      };
      for (int64_t v = threadIdx.x; v < p.nv; v += TPB) {
        const uint4 u = __ldg(p.vec + v);
        each_logit<X>(u, [&](int e, float x) { take(x, p.col0 + uint32_t(v) * Vec<X>::N + e); });
      }
      if (threadIdx.x < p.head + p.tail) {
        const uint32_t col = threadIdx.x < p.head ? threadIdx.x : p.tail_col + threadIdx.x - p.head;
        take(to_f(p.row[col]), col);
      }
      for (int o = 16; o; o >>= 1) {
        const unsigned long long y = __shfl_xor_sync(0xffffffffu, b, o);
        if (y > b) b = y;
      }
      __syncthreads();
      if (lane == 0) s.key[w] = b;
      __syncthreads();
      for (int i = 0; i < WARPS; ++i)
        if (s.key[i] > b) b = s.key[i];
      if (threadIdx.x == 0) s.best[r] = b;
      if (b == 0) break;
      last = b;
    }
  }
  __syncthreads();
}

// ------------------------------------------------------------------------------------------ log probabilities
struct LogprobArgs {
  int64_t V, ld;
  const void* targets;
  int id_type, k;
  float scale;
  int steps;                         // steps of U vectors per group
  float *logprob, *entropy, *lse, *top_logprob;
  int32_t* top_id;
};

struct Sums { float ref, s, st; };   // s = sum 2^t, st = sum 2^t t, both relative to ref (-inf: nothing yet)

// The same sums relative to a larger reference.
__device__ __forceinline__ Sums shift(const Sums& x, float ref, float c2) {
  const float d = ref == x.ref ? 0.0f : max_nan((x.ref - ref) * c2, T_FLOOR);
  const float f = exp2_fast(d);
  return {ref, x.s * f, fmaf(x.s, d, x.st) * f};
}

// The sums of a part whose reference does not fit the fused form (or that is empty): the largest logit first, then the differences.
template <typename X, int TPB>
__device__ __noinline__ Sums sums_of_extremes(const Part<X>& p, float c2, float* sh) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  float m = -INFINITY;
  auto all = [&](auto&& f) {
    if (threadIdx.x < p.head + p.tail) f(to_f(p.row[threadIdx.x < p.head ? threadIdx.x : p.tail_col + threadIdx.x - p.head]));
    for (int64_t v = threadIdx.x; v < p.nv; v += TPB) each_logit<X>(__ldg(p.vec + v), [&](int, float x) { f(x); });
  };
  all([&](float x) { m = fmaxf(m, x); });
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  __syncthreads();
  if (lane == 0) sh[w] = m;
  __syncthreads();
  for (int i = 0; i < TPB / 32; ++i) m = fmaxf(m, sh[i]);
  const float ref = m == -INFINITY ? 0.0f : m;
  Sums x = {m, 0.0f, 0.0f};
  all([&](float v) {
    const float u = max_nan((v - ref) * c2, T_FLOOR), e = exp2_fast(u);
    x.s += e;
    x.st = fmaf(e, u, x.st);
  });
  __syncthreads();
  return x;
}

// A row belongs to a cluster of CTAs (one CTA when there are rows enough), each of which streams a part of it once.
template <typename X, bool TOP, int TPB>
__global__ void __launch_bounds__(TPB, 1024 / TPB) k_token_logprob(const X* __restrict__ logits, const __grid_constant__ LogprobArgs a) {
  constexpr int N = Vec<X>::N, WARPS = TPB / 32;
  extern __shared__ float gmax[];    // [group][thread], with TOP
  __shared__ Sums s_sums[WARPS];
  __shared__ Sums s_part;
  __shared__ TopSmem s_top[1];
  const cg::cluster_group cluster = cg::this_cluster();
  const int ctas = int(cluster.num_blocks()), rank = int(cluster.block_rank());
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t t = blockIdx.x / unsigned(ctas);
  Part<X> p;
  p.row = logits + t * a.ld;
  // the vectors begin at the row's first 16-byte boundary
  const int64_t to16 = int64_t((16 - (reinterpret_cast<uintptr_t>(p.row) & 15)) & 15) / int(sizeof(X));
  const int first = int(min(a.V, to16)), all = (int(a.V) - first) / N, per = (all + ctas - 1) / ctas, v0 = min(all, rank * per);
  p.nv = min(all - v0, per);
  p.vec = reinterpret_cast<const uint4*>(p.row + first) + v0;
  p.col0 = uint32_t(first) + uint32_t(v0) * N;
  p.head = rank == 0 ? uint32_t(first) : 0u;
  p.tail_col = uint32_t(first) + uint32_t(all) * N;
  p.tail = rank == ctas - 1 ? uint32_t(a.V) - p.tail_col : 0u;
  int64_t y = -1;
  float xy = 0.0f;
  if (rank == 0 && threadIdx.x == 0 && a.logprob) {
    y = load_id(a.targets, a.id_type, t, a.V);
    if (y >= 0) xy = to_f(p.row[y]);
  }
  const uint4 none = make_uint4(Vec<X>::NONE, Vec<X>::NONE, Vec<X>::NONE, Vec<X>::NONE);
  const uint4* ptr = p.vec + threadIdx.x;
  const int nv = int(p.nv), n_full = nv / (TPB * U), n_steps = (nv + TPB * U - 1) / (TPB * U);
  auto load = [&](int step, uint4 (&u)[U]) {
    if (step < n_full) {
#pragma unroll
      for (int i = 0; i < U; ++i) u[i] = load_stream(ptr + i * TPB);
    } else {
#pragma unroll
      for (int i = 0; i < U; ++i) u[i] = step * TPB * U + i * TPB + int(threadIdx.x) < nv ? load_stream(ptr + i * TPB) : none;
    }
    ptr += U * TPB;
  };
  const float c2 = a.scale * LOG2E, room = 40.0f / c2;      // a larger logit changes the reference only if it exceeds it by 2^40
  const f2 c22 = pack2(c2, c2);
  float ref = -INFINITY, R = 0.0f, limit = -R_MAX / c2;     // logits below that never set the reference
  f2 minus = pack2(0.0f, 0.0f), s2 = pack2(0.0f, 0.0f), st2 = s2;
  auto raise = [&](float m) {        // a new reference
    const float Rm = m * c2;
    if (ref != -INFINITY) {
      const float d = max_nan(R - Rm, T_FLOOR), f = exp2_fast(d);
      float p0, p1, q0, q1;
      unpack2(s2, p0, p1);
      unpack2(st2, q0, q1);
      p0 += p1;
      s2 = pack2(p0 * f, 0.0f);
      st2 = pack2(fmaf(p0, d, q0 + q1) * f, 0.0f);
    }                                // else nothing but masked logits so far (or a NaN, which stays)
    ref = m;
    R = Rm;
    limit = m + room;
    minus = pack2(-Rm, -Rm);
  };
  auto add_pair = [&](f2 v) {
    float u0, u1;
    unpack2(fma2(v, c22, minus), u0, u1);
    const f2 e = pack2(exp2_fast(u0), exp2_fast(u1));
    s2 = add2(s2, e);
    st2 = fma2(e, pack2(max_nan(u0, T_FLOOR), max_nan(u1, T_FLOOR)), st2);
  };
  float gm = -INFINITY, mine = -INFINITY, extra = -INFINITY;
  int left = a.steps, group = 0;
  auto take = [&](const uint4 (&u)[U]) {
    uint32_t m2 = Vec<X>::max2(Vec<X>::max2(u[0].x, u[0].y), Vec<X>::max2(u[0].z, u[0].w));
#pragma unroll
    for (int i = 1; i < U; ++i) m2 = Vec<X>::max2(m2, Vec<X>::max2(Vec<X>::max2(u[i].x, u[i].y), Vec<X>::max2(u[i].z, u[i].w)));
    const float m = Vec<X>::widen(m2);
    if (m > limit) raise(m);
    mine = fmaxf(mine, m);
    if (TOP) {
      gm = fmaxf(gm, m);
      if (--left == 0) {
        gmax[group++ * TPB + threadIdx.x] = gm;
        gm = -INFINITY;
        left = a.steps;
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int j = 0; j < N / 2; ++j) add_pair(Vec<X>::pair(u[i], j));
  };
  uint4 even[U], odd[U];
  if (n_steps > 0) load(0, even);
  if (threadIdx.x < p.head + p.tail) {
    extra = to_f(p.row[threadIdx.x < p.head ? threadIdx.x : p.tail_col + threadIdx.x - p.head]);
    if (extra > limit) raise(extra);
    add_pair(pack2(extra, -INFINITY));
  }
  for (int step = 0; step < n_steps; step += 2) {
    if (step + 1 < n_steps) load(step + 1, odd);
    take(even);
    if (step + 1 >= n_steps) break;
    if (step + 2 < n_steps) load(step + 2, even);
    take(odd);
  }
  if (TOP && left != a.steps) gmax[group++ * TPB + threadIdx.x] = gm;
  Sums x;
  {
    float p0, p1, q0, q1;
    unpack2(s2, p0, p1);
    unpack2(st2, q0, q1);
    const float d = ref == -INFINITY ? 0.0f : fmaf(ref, c2, -R), f = 1.0f - LN2 * d;      // d: at most half a unit of R; 2^-d
    x = {ref, (p0 + p1) * f, fmaf(-d, p0 + p1, q0 + q1) * f};
  }
  const float top = fmaxf(mine, extra);
  // logits that the fused form cannot take: too large ones anywhere, or nothing but too small ones
  if (__syncthreads_or(top * c2 > R_MAX) || (!__syncthreads_or(ref != -INFINITY) && __syncthreads_or(top > -INFINITY)))
    x = sums_of_extremes<X, TPB>(p, c2, &s_sums[0].ref);
  // the threads' sums to one reference, warp by warp and then together
  float m = x.ref;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  x = shift(x, m, c2);
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
    x.st += __shfl_xor_sync(0xffffffffu, x.st, o);
  }
  if (lane == 0) s_sums[w] = x;
  __syncthreads();
  x = s_sums[lane % WARPS];
  m = x.ref;
#pragma unroll
  for (int o = WARPS / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  x = shift(x, m, c2);
#pragma unroll
  for (int o = WARPS / 2; o; o >>= 1) {
    x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
    x.st += __shfl_xor_sync(0xffffffffu, x.st, o);
  }
  if (TOP) best_of_part<X, TPB>(p, a.k, gmax, group, a.steps, mine, s_top[0]);
  if (ctas > 1) {
    if (threadIdx.x == 0) s_part = x;
    cluster.sync();
    if (rank == 0) {
      x = *cluster.map_shared_rank(&s_part, unsigned(lane % ctas));
      m = x.ref;
      for (int o = ctas / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      x = shift(x, m, c2);
      for (int o = ctas / 2; o; o >>= 1) {
        x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
        x.st += __shfl_xor_sync(0xffffffffu, x.st, o);
      }
      if (TOP) {
        for (int i = threadIdx.x; i < ctas * a.k; i += TPB) s_top[0].key[i] = cluster.map_shared_rank(&s_top[0], unsigned(i / a.k))->best[i % a.k];
        __syncthreads();
        if (threadIdx.x < MV_TOP_MAX) s_top[0].best[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < ctas * a.k; i += TPB) {
          const unsigned long long mykey = s_top[0].key[i];
          if (mykey == 0) continue;
          int place = 0;
          for (int j = 0; j < ctas * a.k; ++j) place += s_top[0].key[j] > mykey;
          if (place < a.k) s_top[0].best[place] = mykey;
        }
        __syncthreads();
      }
    }
    cluster.sync();                  // the parts stay until they have been read
    if (rank != 0) return;
  }
  const bool empty = x.s == 0.0f;
  const float r = empty ? 0.0f : x.ref, ls = logf(x.s);
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[t] = empty ? -INFINITY : fmaf(a.scale, r, ls);
    if (a.entropy) a.entropy[t] = empty ? 0.0f : ls - LN2 * (x.st / x.s);
    if (a.logprob) a.logprob[t] = y < 0 ? 0.0f : empty ? -INFINITY : (xy - r) * a.scale - ls;
  }
  if (TOP && int(threadIdx.x) < a.k) {
    const unsigned long long key = s_top[0].best[threadIdx.x];
    const float v = key_value(key);
    if (a.top_id) a.top_id[t * a.k + threadIdx.x] = key ? int32_t(key_index(key)) : -1;
    if (a.top_logprob) a.top_logprob[t * a.k + threadIdx.x] = isnan(x.s) ? x.s : key == 0 || v == -INFINITY ? -INFINITY : (v - r) * a.scale - ls;
  }
}

constexpr int GRAD_TPB = 256;

template <typename X>
__global__ void __launch_bounds__(GRAD_TPB) k_token_grad(const X* logits, int64_t V, int64_t ld, const void* __restrict__ targets, int id_type, float scale,
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
  for (int64_t j = threadIdx.x; j < V; j += GRAD_TPB) {
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
  LogprobArgs a;
  a.V = V; a.ld = ld; a.targets = targets; a.id_type = id_type; a.k = k; a.scale = scale;
  a.logprob = logprob; a.entropy = entropy; a.lse = lse; a.top_logprob = top_logprob; a.top_id = top_id;
  return with_type(type, [&](auto x) {
    using X = decltype(x);
    const int64_t vecs = V / Vec<X>::N;
    // Many rows: small CTAs, whose ends overlap with the others' streaming.  Fewer rows than multiprocessors: large CTAs, and as many per row
    // (up to the eight of a portable cluster) as keep a whole step for each thread and fit the device at once.
    const int tpb = T < 148 ? 512 : 128;
    int ctas = 1;
    while (ctas < 8 && T * ctas * tpb < 148 * 1024 && vecs >= int64_t(ctas) * 2 * tpb * U) ctas *= 2;
    const int64_t n_steps = ((vecs + ctas - 1) / ctas + tpb * U - 1) / (tpb * U);
    a.steps = int((n_steps + MAX_GROUPS - 1) / MAX_GROUPS);
    if (a.steps < 1) a.steps = 1;
    if (T * ctas >= lim) return int(MV_ERR_INVALID_ARG);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(T * ctas));
    cfg.blockDim = dim3(unsigned(tpb));
    cfg.dynamicSmemBytes = k ? size_t((n_steps + a.steps - 1) / a.steps) * tpb * 4 : 0;
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = unsigned(ctas);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    auto* kernel = tpb == 128 ? (k ? k_token_logprob<X, true, 128> : k_token_logprob<X, false, 128>)
                              : (k ? k_token_logprob<X, true, 512> : k_token_logprob<X, false, 512>);
    if (cfg.dynamicSmemBytes > 32 << 10 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 64 << 10) != cudaSuccess) {
      cudaGetLastError();
      return int(MV_ERR_CUDA);
    }
    const bool ok = cudaLaunchKernelEx(&cfg, kernel, static_cast<const X*>(logits), a) == cudaSuccess;
    return cuda_ok() == MV_OK && ok ? int(MV_OK) : int(MV_ERR_CUDA);
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
    k_token_grad<X><<<unsigned(T), GRAD_TPB, 0, st>>>(static_cast<const X*>(logits), V, ld, targets, id_type, scale, lse, entropy, g_logprob, g_entropy,
                                                  static_cast<X*>(dlogits), ldg);
    return cuda_ok();
  });
}

}  // extern "C"
