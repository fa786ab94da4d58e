// mv_token.cu -- log probabilities of given tokens with entropy and alternatives, and their gradient, for sm_100a.
//
// The exponentials and their sums are in mv_row.cuh.

#include "mv_row.cuh"

namespace {

// ------------------------------------------------------------------------------------------ alternatives
// The k largest logits cost the streaming pass almost nothing: a thread keeps the largest logit of every group (a few
// vectors) that it reads.  Afterwards a bound B is found that at least k group maxima reach; every logit above B lies in a
// group whose maximum is above B, and those few groups are read again.
constexpr int U = 4;                 // vectors per thread and step, all in flight, two by two from neighbouring places
constexpr int MAX_GROUPS = 32;       // groups per thread

template <int TPB> struct TopSmem {
  static constexpr int GROUP_LIST = 256;                    // groups read again
  static constexpr int KEY_LIST = TPB >= 128 ? 1024 : 256;  // candidates
  unsigned long long key[KEY_LIST];
  unsigned long long best[MV_TOP_MAX];
  uint16_t group[GROUP_LIST];
  float sorted[TPB / 32][32];        // of each warp
  float bound;
  int n_key, n_group, found;
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

template <int TPB> __device__ __forceinline__ void push_key(TopSmem<TPB>& s, float x, uint32_t col) {
  const int i = atomicAdd(&s.n_key, 1);
  if (i < s.KEY_LIST) s.key[i] = make_key(x, col);
}

// Every candidate's place is the number of candidates before it.
template <int TPB> __device__ __forceinline__ void rank_keys(TopSmem<TPB>& s, int n, int k) {
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += TPB) {
    const unsigned long long mine = s.key[i];
    int place = 0;
#pragma unroll 2
    for (int j = 0; j < n; ++j) place += s.key[j] > mine;
    if (place < k && mine != 0) s.best[place] = mine;
  }
}

// The elements of the listed groups that reach the bound (or lie above it) become candidates.
template <typename X, int TPB> __device__ __forceinline__ void gather_groups(const Part<X>& p, int listed, int steps, bool above, TopSmem<TPB>& s) {
  const float B = s.bound;
  const unsigned per = unsigned(steps) * U;                          // vectors per group
#pragma unroll 1
  for (unsigned i = threadIdx.x; i < listed * per; i += TPB) {
    const unsigned q = steps == 1 ? i / U : i / per, gi = s.group[q], j = i - q * per, v = 2 * (gi % TPB + (gi / TPB * (per / 2) + j / 2) * TPB) + j % 2;
    if (int64_t(v) >= p.nv) continue;
    const uint4 u = __ldg(p.vec + v);
    unsigned hit = 0;
    each_logit<X>(u, [&](int e, float y) { hit |= (above ? y > B : y >= B) ? 1u << e : 0u; });
    for (; hit; hit &= hit - 1) {
      const unsigned c = v * Vec<X>::N + __ffs(int(hit)) - 1;
      push_key(s, to_f(reinterpret_cast<const X*>(p.vec)[c]), p.col0 + c);
    }
  }
}

// The groups whose maximum reaches the bound (or lies above it).
template <int TPB> __device__ __forceinline__ void list_groups(const float* gmax, int groups, bool above, TopSmem<TPB>& s) {
  const float B = s.bound;
#pragma unroll 1
  for (int g0 = 0; g0 < groups; g0 += 8) {
    float m[8];
#pragma unroll
    for (int g = 0; g < 8; ++g) m[g] = g0 + g < groups ? gmax[(g0 + g) * TPB + threadIdx.x] : -INFINITY;
    unsigned hit = 0;
#pragma unroll
    for (int g = 0; g < 8; ++g) hit |= g0 + g < groups && (above ? m[g] > B : m[g] >= B) ? 1u << g : 0u;
    if (hit == 0) continue;
    int i = atomicAdd(&s.n_group, __popc(hit));
    for (; hit; hit &= hit - 1, ++i)
      if (i < s.GROUP_LIST) s.group[i] = uint16_t((g0 + __ffs(int(hit)) - 1) * TPB + threadIdx.x);
  }
}

// Rows with crowds: many groups at the bound itself (few distinct values; fewer logits than k left by a mask), or large
// logits crowded in the columns of few threads.  Not inlined: seldom run.
template <typename X, int TPB>
__device__ __noinline__ void best_of_crowd(const Part<X>& p, int k, const float* gmax, int groups, int steps, float mine, TopSmem<TPB>& s) {
  constexpr int WARPS = TPB / 32;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const float B = s.bound;
  const X* x = reinterpret_cast<const X*>(p.vec);
  const uint32_t n = uint32_t(p.nv) * Vec<X>::N;
  auto ends = [&](auto&& f) {
    if (threadIdx.x < p.head + p.tail) {
      const uint32_t col = threadIdx.x < p.head ? threadIdx.x : p.tail_col + threadIdx.x - p.head;
      f(to_f(p.row[col]), col);
    }
  };
  __syncthreads();
  if (threadIdx.x == 0) { s.n_key = 0; s.n_group = 0; s.found = 0; }
  __syncthreads();
  ends([&](float v, uint32_t col) { if (v == v) push_key(s, v, col); });
  if (mine > B) list_groups<TPB>(gmax, groups, true, s);
  __syncthreads();
  const int above = s.n_group;
  gather_groups<X, TPB>(p, min(above, s.GROUP_LIST), steps, true, s);
  __syncthreads();
  bool whole = above <= s.GROUP_LIST && s.n_key <= s.KEY_LIST;
  if (whole) {
    // the logits at the bound, in order from the start of the part until k of them are found (they are many)
#pragma unroll 1
    for (uint32_t c0 = 0; c0 < n; c0 += TPB * 8) {
      const uint32_t c1 = c0 + threadIdx.x * 8;
      unsigned hit = 0;
      for (uint32_t e = 0; e < 8; ++e)
        if (c1 + e < n && to_f(x[c1 + e]) == B) hit |= 1u << e;
      int incl = __popc(hit);
      for (int o = 1; o < 32; o <<= 1) {
        const int z = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += z;
      }
      if (lane == 31) s.sorted[w][0] = __int_as_float(incl);
      __syncthreads();
      int at = s.found + incl - __popc(hit), all = s.found;
      for (int i = 0; i < WARPS; ++i) {
        const int c = __float_as_int(s.sorted[i][0]);
        at += i < w ? c : 0;
        all += c;
      }
      for (uint32_t e = 0; e < 8; ++e)
        if ((hit >> e & 1u) && at++ < k) push_key(s, B, p.col0 + c1 + e);
      __syncthreads();
      if (threadIdx.x == 0) s.found = all;
      __syncthreads();
      if (all >= k) break;
    }
    whole = s.n_key <= s.KEY_LIST;
  }
  if (whole) {
    rank_keys<TPB>(s, s.n_key, k);
  } else {
    // one reading of the part per alternative
    unsigned long long last = ~0ull;
#pragma unroll 1
    for (int r = 0; r < k; ++r) {
      unsigned long long b = 0;
      auto take = [&](float v, uint32_t col) {
        const unsigned long long y = v == v ? make_key(v, col) : 0;
        if (y < last && y > b) b = y;
      };
      for (uint32_t c = threadIdx.x; c < n; c += TPB) take(to_f(x[c]), p.col0 + c);
      ends(take);
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
}

// What the choice of the best needs before the next barrier.
template <int TPB> __device__ __forceinline__ void begin_best(float mine, TopSmem<TPB>& s) {
  s.sorted[threadIdx.x >> 5][threadIdx.x & 31] = sort_warp(mine);
  if (threadIdx.x == 0) { s.n_key = 0; s.n_group = 0; }
  for (int i = threadIdx.x; i < MV_TOP_MAX; i += TPB) s.best[i] = 0;
}

// The k best keys of this part, in order, in s.best (0 where there are fewer).  All threads; ends with a barrier.
template <typename X, int TPB>
__device__ __forceinline__ void best_of_part(const Part<X>& p, int k, const float* gmax, int groups, int steps, float mine, TopSmem<TPB>& s) {
  constexpr int WARPS = TPB / 32;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  // the single logits at the ends are always candidates
  if (threadIdx.x < p.head + p.tail) {
    const uint32_t col = threadIdx.x < p.head ? threadIdx.x : p.tail_col + threadIdx.x - p.head;
    const float x = to_f(p.row[col]);
    if (x == x) push_key(s, x, col);
  }
  if (w == 0) {
    // If j warps hold r maxima >= b each, j r >= k of them reach b: lane r - 1 tries r, with the ceil(k / r)-th largest of the warps' r-th maxima.
    float v[WARPS], b = -INFINITY;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) v[i] = s.sorted[i][lane];
    const int j = (k + lane) / (lane + 1);
#pragma unroll 1
    for (int i = 0; i < WARPS; ++i) {
      const float vi = s.sorted[i][lane];
      int reach = 0;
#pragma unroll
      for (int m = 0; m < WARPS; ++m) reach += v[m] >= vi;
      if (reach >= j) b = fmaxf(b, vi);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) b = fmaxf(b, __shfl_xor_sync(0xffffffffu, b, o));
    if (lane == 0) s.bound = b;
  }
  __syncthreads();
  if (mine >= s.bound) list_groups<TPB>(gmax, groups, false, s);
  __syncthreads();
  const int listed = s.n_group;
  if (listed <= s.GROUP_LIST) gather_groups<X, TPB>(p, listed, steps, false, s);
  __syncthreads();
  const int n = s.n_key;
  if (listed <= s.GROUP_LIST && n <= s.KEY_LIST) rank_keys<TPB>(s, n, k);
  else best_of_crowd<X, TPB>(p, k, gmax, groups, steps, mine, s);
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

// A row belongs to a CTA (to a cluster of CTAs when there are few), each of which streams its part once, two steps of 64 bytes a
// lane on their way.  Per 16 bytes of bf16 a lane spends about 40 instructions, eight of them exponentials, which the
// multiprocessor does at 16 a cycle against the 11.4 logits a cycle that memory brings: so issue, the exponentials and memory
// are all within a factor of two of one another, and under the power limit (1.68 GHz in a long run) the instructions count.
// 8192 x 65536 bf16: 176 us without alternatives (6.1 TB/s), 191 us with 16 of them (207 us at the limit); the
// alternatives' cost is the end of a row, about 2 us of latency that the other CTAs of the multiprocessor only partly cover.
// Rows that are summed again by differences cost a second, plainer reading: 450 us without alternatives, 485 us with them.
template <typename X, bool TOP, int TPB>
__global__ void __launch_bounds__(TPB, 1024 / TPB) k_token_logprob(const X* __restrict__ logits, const __grid_constant__ LogprobArgs a) {
  constexpr int N = Vec<X>::N, WARPS = TPB / 32;
  extern __shared__ float gmax[];    // [group][thread], with TOP
  __shared__ Sums s_sums[WARPS];
  __shared__ Sums s_part;
  __shared__ TopSmem<TPB> s_top[1];
  const cg::cluster_group cluster = cg::this_cluster();
  const int ctas = int(cluster.num_blocks()), rank = int(cluster.block_rank());
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t t = ctas == 1 ? blockIdx.x : blockIdx.x / unsigned(ctas);
  Part<X> p;
  p.row = logits + t * a.ld;
  // the vectors begin at the row's first 32-byte boundary
  const int64_t to32 = int64_t((32 - (reinterpret_cast<uintptr_t>(p.row) & 31)) & 31) / int(sizeof(X));
  const int first = int(min(a.V, to32)), all = (int(a.V) - first) / (2 * N) * 2, per = (all / 2 + ctas - 1) / ctas * 2, v0 = min(all, rank * per);
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
  const uint4* ptr = p.vec + 2 * threadIdx.x;
  const int nv = int(p.nv), n_full = nv / (TPB * U), n_steps = (nv + TPB * U - 1) / (TPB * U);
  auto load = [&](int step, uint4 (&u)[U]) {
    if (step < n_full) {
#pragma unroll
      for (int i = 0; i < U; i += 2) load_stream(ptr + i * TPB, u[i], u[i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < U; i += 2) {
        u[i] = u[i + 1] = none;
        if ((step * U + i) * TPB + 2 * int(threadIdx.x) < nv) load_stream(ptr + i * TPB, u[i], u[i + 1]);
      }
    }
    ptr += U * TPB;
  };
  const float c2 = fminf(a.scale * LOG2E, 3.0e38f), room = LAG / c2;
  const f2 c22 = pack2(c2, c2);
  // logits below the first limit never set the reference; beside a reference above -R_MAX their 2^t is 0
  float ref = -INFINITY, R = 0.0f, limit = -2.0f * R_MAX / c2;
  // bf16 has the range of 32 bits: two logits at a time are kept above a floor so far below the limit that 2^t is 0 there,
  // and so near that t is finite; for the other types t itself is kept above T_FLOOR
  constexpr bool FLOOR2 = sizeof(X) == 2 && Vec<X>::NONE == 0xff80ff80u;
  uint32_t floor2 = 0;
  if constexpr (FLOOR2) floor2 = (__float_as_uint(fmaxf(-8.0f * R_MAX / c2, -3.0e38f)) >> 16) * 0x10001u;
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
    if constexpr (!FLOOR2) st2 = fma2(e, pack2(max_nan(u0, T_FLOOR), max_nan(u1, T_FLOOR)), st2);
    else st2 = fma2(e, pack2(u0, u1), st2);
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
    for (int i = 0; i < U; ++i) {
      uint4 v = u[i];
      if constexpr (FLOOR2) v = make_uint4(Vec<X>::max2_nan(v.x, floor2), Vec<X>::max2_nan(v.y, floor2), Vec<X>::max2_nan(v.z, floor2), Vec<X>::max2_nan(v.w, floor2));
#pragma unroll
      for (int j = 0; j < N / 2; ++j) add_pair(Vec<X>::pair(v, j));
    }
  };
  uint4 even[U], odd[U];
  if (n_steps > 0) load(0, even);
  if (threadIdx.x < p.head + p.tail) {
    extra = to_f(p.row[threadIdx.x < p.head ? threadIdx.x : p.tail_col + threadIdx.x - p.head]);
    if (extra > limit) raise(extra);
    add_pair(pack2(FLOOR2 ? max_nan(extra, __uint_as_float(floor2 << 16)) : extra, __uint_as_float(FLOOR2 ? floor2 << 16 : 0xff800000u)));
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
    const float d = ref == -INFINITY ? 0.0f : fmaf(ref, c2, -R), f = fmaf(fmaf(0.5f * LN2 * LN2, d, -LN2), d, 1.0f);      // d: at most half a unit of R; 2^-d
    x = {ref, (p0 + p1) * f, fmaf(-d, p0 + p1, q0 + q1) * f};
  }
  const float top = fmaxf(mine, extra);
  // the sums of `width` neighbouring lanes to one reference, at least m: the largest logit, so that log s is not negative
  auto fold = [&](int width, float m) {
    m = fmaxf(m, x.ref);
#pragma unroll
    for (int o = width / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    x = shift(x, m, c2);
#pragma unroll
    for (int o = width / 2; o; o >>= 1) {
      x.s += __shfl_xor_sync(0xffffffffu, x.s, o);
      x.st += __shfl_xor_sync(0xffffffffu, x.st, o);
    }
  };
  fold(32, top);
  if (lane == 0) s_sums[w] = x;
  if (TOP) begin_best(mine, s_top[0]);
  const bool large = __syncthreads_or(top * c2 > R_MAX);
  x = s_sums[lane % WARPS];
  fold(WARPS, -INFINITY);
  // logits that the fused form cannot take: too large ones anywhere, or none that is not too low (x.ref: the largest of all)
  if (large || c2 < C2_MIN || (x.ref * c2 < -R_MAX && x.ref > -INFINITY)) {
    x = sums_of_extremes<X, TPB>(p, c2, top, &s_sums[0].ref);
    fold(32, -INFINITY);
    if (lane == 0) s_sums[w] = x;
    __syncthreads();
    x = s_sums[lane % WARPS];
    fold(WARPS, -INFINITY);
  }
  if (TOP) best_of_part<X, TPB>(p, a.k, gmax, group, a.steps, mine, s_top[0]);
  if (ctas > 1) {
    if (threadIdx.x == 0) s_part = x;
    cluster.sync();
    if (rank == 0) {
      x = *cluster.map_shared_rank(&s_part, unsigned(lane % ctas));
      fold(ctas, -INFINITY);
      if (TOP) {
        for (int i = threadIdx.x; i < ctas * a.k; i += TPB) s_top[0].key[i] = cluster.map_shared_rank(&s_top[0], unsigned(i / a.k))->best[i % a.k];
        __syncthreads();
        for (int i = threadIdx.x; i < MV_TOP_MAX; i += TPB) s_top[0].best[i] = 0;
        __syncthreads();
        rank_keys<TPB>(s_top[0], ctas * a.k, a.k);
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
    if (a.logprob) a.logprob[t] = y < 0 ? 0.0f : empty ? -INFINITY : distance(xy, r, a.scale) - ls;
  }
  if (TOP)
    for (int i = threadIdx.x; i < a.k; i += TPB) {
      const unsigned long long key = s_top[0].best[i];
      const float v = key_value(key);
      if (a.top_id) a.top_id[t * a.k + i] = key ? int32_t(key_index(key)) : -1;
      if (a.top_logprob) a.top_logprob[t * a.k + i] = isnan(x.s) ? x.s : key == 0 || v == -INFINITY ? -INFINITY : distance(v, r, a.scale) - ls;
    }
}

// ------------------------------------------------------------------------------------------ gradient
// dx = c (g1 (1[v = y] - p) - g2 p (log p + H)), log p = c x - lse.  With h = log2(p) / 2 and q = 2^h:
// dx = q (q (A h + B)) + c g1 1[v = y], A = -2 ln 2 c g2, B = -c (g1 + g2 H): two fused multiply-adds, an exponential and three
// products per logit.  The difference c x - lse is taken first, in one rounding: two products of its terms with log2(e) would
// differ by their own roundings, which for an lse of 1e9 are tens; and since the lse itself is rounded by as much there, log p is kept
// from being positive (4096 x 131072 bf16: 358 us, without that 355.5; asking it only of rows with a large lse: 358).  p is formed
// as q q because the hardware's exponential has no subnormal results; that doubles its error to 2^-21, beside the 2^-11 (f16) or
// 2^-8 (bf16) of the result's rounding.  Each CTA takes one stretch of one row, so that the stretches, in the order of memory, go
// to the multiprocessors as they become free: memory bounds it (6.0 TB/s in and out; 365 us with the power limit reached, in a
// long run).  Where logits and gradient lie differently within 16 bytes, single elements are read and written: 1041 us.
constexpr int GRAD_TPB = 256, GRAD_U = 4;
constexpr float H_FLOOR = -256.0f;     // q is 0 from -127 on; so near that A h is finite for any gradient below 1e36

struct GradArgs {
  int64_t V, ld, ldg;
  const void* targets;
  int id_type;
  float scale;
  unsigned stretches;                // CTAs per row
  const float *lse, *entropy, *g_logprob, *g_entropy;
};

// VEC: logits and gradient start at the same place within 16 bytes in every row.
template <typename X, bool VEC>
__global__ void __launch_bounds__(GRAD_TPB) k_token_grad(const X* logits, X* dlogits, const __grid_constant__ GradArgs a) {
  constexpr int N = Vec<X>::N;
  const int64_t t = blockIdx.x / a.stretches;
  const unsigned stretch = blockIdx.x % a.stretches;
  const X* x = logits + t * a.ld;
  X* dx = dlogits + t * a.ldg;
  const int64_t y = a.targets ? load_id(a.targets, a.id_type, t, a.V) : -1;
  const float l = a.lse[t];
  const float g1 = y >= 0 && a.g_logprob ? a.g_logprob[t] : 0.0f;
  const float g2 = a.g_entropy ? a.g_entropy[t] : 0.0f;
  const bool none = (g1 == 0.0f && g2 == 0.0f) || l == -INFINITY;
  const float sum = g1 + (g2 == 0.0f ? 0.0f : g2 * a.entropy[t]);
  const float l2e = 0.5f * LOG2E, A = -2.0f * LN2 * a.scale * g2, B = -a.scale * sum;
  auto one = [&](float v, int64_t col) {      // the same operations as two logits at a time below: a row's bits do not depend on its place
    if (none) return 0.0f;
    const float h = min_nan(max_nan(fmaf(v, a.scale, -l) * l2e, H_FLOOR), 0.0f), q = exp2_fast(h), d = q * (q * fmaf(h, A, B));
    return col == y ? fmaf(a.scale, g1, d) : d;
  };
  // the vectors begin at the row's first 16-byte boundary; what is before and behind them goes to the first stretch
  const int64_t first = VEC ? min(a.V, int64_t((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / int(sizeof(X))) : 0;
  const int64_t nv = VEC ? (a.V - first) / N : 0;
  if (VEC && stretch == 0) {
    const int64_t behind = first + nv * N;
    if (int64_t(threadIdx.x) < first + a.V - behind) {
      const int64_t col = int64_t(threadIdx.x) < first ? int64_t(threadIdx.x) : behind + threadIdx.x - first;
      dx[col] = from_f<X>(one(to_f(x[col]), col));
    }
  }
  if constexpr (VEC) {
    const int64_t v0 = int64_t(stretch) * GRAD_TPB * GRAD_U + threadIdx.x;
    const uint4* in = reinterpret_cast<const uint4*>(x + first);
    uint4* out = reinterpret_cast<uint4*>(dx + first);
    if (none) {
#pragma unroll
      for (int i = 0; i < GRAD_U; ++i)
        if (v0 + i * GRAD_TPB < nv) __stcs(out + v0 + i * GRAD_TPB, make_uint4(0, 0, 0, 0));
      return;
    }
    const f2 scale2 = pack2(a.scale, a.scale), minus = pack2(-l, -l), l2e2 = pack2(l2e, l2e), A2 = pack2(A, A), B2 = pack2(B, B);
    uint4 u[GRAD_U];
#pragma unroll
    for (int i = 0; i < GRAD_U; ++i)
      if (v0 + i * GRAD_TPB < nv) u[i] = __ldcs(in + v0 + i * GRAD_TPB);
#pragma unroll
    for (int i = 0; i < GRAD_U; ++i) {
      const int64_t v = v0 + i * GRAD_TPB;
      if (v >= nv) break;
      float d[N];
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        float h0, h1;
        unpack2(mul2(fma2(Vec<X>::pair(u[i], j), scale2, minus), l2e2), h0, h1);
        h0 = min_nan(max_nan(h0, H_FLOOR), 0.0f);
        h1 = min_nan(max_nan(h1, H_FLOOR), 0.0f);
        const f2 q = pack2(exp2_fast(h0), exp2_fast(h1));
        unpack2(mul2(q, mul2(q, fma2(pack2(h0, h1), A2, B2))), d[2 * j], d[2 * j + 1]);
      }
      const int64_t hot = y - first - v * N;
      if (hot >= 0 && hot < N) {     // the target's term belongs inside the sum that is rounded
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (e == hot) d[e] = one(to_f(x[first + v * N + e]), y);
      }
      __stcs(out + v, pack_vec<X>(d));
    }
  } else {
    const int64_t c0 = int64_t(stretch) * GRAD_TPB * GRAD_U * N, c1 = min(a.V, c0 + GRAD_TPB * GRAD_U * N);
    for (int64_t c = c0 + threadIdx.x; c < c1; c += GRAD_TPB) dx[c] = from_f<X>(one(to_f(x[c]), c));
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
    // A CTA per row.  Its end (choosing the alternatives) is a chain of short phases, so short rows take few threads and many
    // CTAs, if there are rows enough to fill the device: 16000 rows of 16 KB, k = 8: 62 us with 32 threads, 73 with 64, 102 with 128;
    // 9079 rows of 33 KB: 77, 70, 84; with 64 and 128, 8000 of 48 KB: 79 and 84, of 64 KB: 103 and 103 to 105.  Rows in the hundreds take more threads than that (1003 of 16 KB: 10.4, 9.5, 9.6), long ones
    // more still (3000 of 131 KB: 81 us with 128, 86 with 256; of 200 KB: 136 and 123; 100 of 200 KB: 14.4 and 11.3).
    // Long rows that are so few that four CTAs each fit the device: a cluster of four per row, a step or more for each thread (one
    // row of 200 KB: 8.8 us, with one CTA 10.3; 32 of 262 KB: 9.5 and 14.0).
    // 32 threads have too few maxima to bound more than 32 alternatives.
    const int tpb = T >= 2368 && vecs <= 2047 && k <= 32 ? 32
                  : T >= 1184 && vecs <= 3000 ? 64
                  : vecs > 10240 || (T < 600 && vecs > 6000) ? 256 : 128;
    const int ctas = T <= 148 / 4 && vecs >= 4 * 256 * U ? 4 : 1;
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
    cfg.numAttrs = ctas > 1;
    auto pick = [&](auto top) {
      constexpr bool TOP = decltype(top)::value;
      return tpb == 32 ? k_token_logprob<X, TOP, 32> : tpb == 64 ? k_token_logprob<X, TOP, 64>
           : tpb == 128 ? k_token_logprob<X, TOP, 128> : k_token_logprob<X, TOP, 256>;
    };
    auto* kernel = k ? pick(std::true_type()) : pick(std::false_type());
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
  if (share_bytes(logits, T, V, ld, type_size(type), dlogits, T, V, ldg, type_size(type)) && !(logits == dlogits && ld == ldg))
    return MV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_type(type, [&](auto x) {
    using X = decltype(x);
    GradArgs g;
    g.V = V; g.ld = ld; g.ldg = ldg; g.targets = targets; g.id_type = id_type; g.scale = scale;
    g.lse = lse; g.entropy = entropy; g.g_logprob = g_logprob; g.g_entropy = g_entropy;
    const int64_t per = int64_t(GRAD_TPB) * GRAD_U * Vec<X>::N, stretches = (V + per - 1) / per;
    if (T * stretches >= lim) return int(MV_ERR_INVALID_ARG);
    g.stretches = unsigned(stretches);
    // a gradient that lies otherwise within 16 bytes than the logits, in some row, is written one by one
    const bool vec = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(dlogits)) & 15) == 0 &&
                     (T == 1 || (ld - ldg) * int64_t(sizeof(X)) % 16 == 0);
    auto* kernel = vec ? k_token_grad<X, true> : k_token_grad<X, false>;
    kernel<<<unsigned(T * stretches), GRAD_TPB, 0, st>>>(static_cast<const X*>(logits), static_cast<X*>(dlogits), g);
    return cuda_ok();
  });
}

}  // extern "C"
