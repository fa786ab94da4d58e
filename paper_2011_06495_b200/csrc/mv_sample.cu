// mv_sample.cu -- one token per row from softmax(scale * logits), cut to the top k, the top p and the min p, for sm_100a.
//
// Whether a token stays, and which one is drawn, hangs on where a sum of weights passes a limit; with 10^5 tokens the borders between
// them lie 10^-5 of the sum apart and less, so weights are formed in 64 bits.  They are added as whole numbers, the largest being 2^61 / V
// (V rounded up to a power of two, at least 1024): sums are exact and do not depend on the order in which they are formed.
//
// A CTA, or a cluster of two to eight where there are few rows, reads its row once for the largest logit, and then, by request:
//   top k up to 1024           the maxima of groups of tokens give a bound that the top k reach; the tokens beyond it (some more than k)
//                              are listed, sorted, summed up, cut, and drawn from.  One row of 131072 bf16: 12 us, 256 rows 34 (greedy) to
//                              38; what is not the reading is a chain of short phases, about 8 us.
//   nothing, min p             one more reading (out of L2), 64-bit weights summed by chunks of 512 tokens; the chunk where the limit is
//                              passed is read again.  256 rows of 131072 bf16 67 us, 1024 of 50021 f32 102: 28 and 43 us of it 64-bit
//                              arithmetic, the rest the two readings, one after the other in every CTA.
//   top p, or a larger top k   a count by 4096 bins of the logits first, which bounds where the cut lies, then the same reading with a list of
//                              the tokens there.  One row 38 us, 256 rows 156.  Where too many lie there (16-bit logits far from zero: a few
//                              values), a third reading; 64 rows of 131072 bf16 around 10: 127 us.
// What none of these takes goes to a plain form with exact cuts by radix, ten readings or more by one CTA, the others of its row gone:
//   top k and top p together where the list overflows or k is above 1024: one row of 131072 f32, top k 2000 and top p 0.9, 1.5 ms, 64 rows 1.9; equal
//                              logits meet in one bin, 131072 of them (a constant row, top k 50 and top p 0.9) 34 ms, 64 such rows 40
//   logits beyond 2^20 times a unit of the softmax (inverse temperatures of 10^5 and more; or below 10^-36): one row 0.34 ms, 64 rows 0.57, greedy 1.0
//   more than 1 043 000 tokens, unless the top k are listed: 4 rows of 1 500 000 bf16 3.0 ms, with top p 15 (of 1 000 000: 43 us and 0.2 ms)
//   any other crowd that two passes of narrowing leave of more than one value
// Times are those of calls that follow one another for half a second.

#include "mv_row.cuh"

namespace {

typedef unsigned long long u64;
template <int I> using Int = std::integral_constant<int, I>;

struct SampleArgs {
  int64_t V, ld;
  const float *u, *scale, *top_p, *min_p;
  const int32_t* top_k;
  double unit;                       // whole numbers that the largest weight is
  void* token;
  int id_type;
  float* logprob;
  int steps;                         // steps of U vectors per group
  int chunks;                        // chunks of the row, its ends included; 0: too many for the fast paths
};

// The order of the logits as that of 32-bit numbers: larger is earlier; +0 and -0 are one value.  A key is an order and, below it, the
// index, lower ones first.
__device__ __forceinline__ uint32_t order_of(float x) { return uint32_t(make_key(x, 0) >> 32); }
__device__ __forceinline__ float value_of(uint32_t h) { return key_value(u64(h) << 32); }

constexpr int TPB = 256, WARPS = TPB / 32, U = 4;
constexpr int LIST = 1024;           // candidates
constexpr int CHUNKS = 2048;         // sums over neighbouring tokens
constexpr int CHUNK = 512;           // tokens of each, 16 neighbouring ones for each lane of a warp
constexpr int GROUPS = 32;           // groups per thread whose maxima are kept
constexpr int COARSE = 512, FINE = 4096;       // bins over 2^-32 .. 1 of the largest weight: 1/16 and 1/128 of a power of two wide
constexpr int SLOW_BINS = 2048;
constexpr int TABLE = 16;
constexpr int RESIDENT = 4;          // CTAs per multiprocessor
constexpr int MOST_CTAS = 8;         // per row

// What a row's request asks for.
struct Request {
  float u, scale, p, mp;
  int64_t k;
  bool valid;
};

// What one path or the other keeps in shared memory.
struct Smem {
  union {
    float gmax[GROUPS][TPB];         // the groups' maxima
    struct {
      union {
        uint32_t bin[FINE];
        struct { u64 sorted[LIST], sum[LIST]; };
      };
      u64 chunk[CHUNKS];
    } fast;
    struct {
      u64 bin[SLOW_BINS];
      u64 chunk[CHUNKS];
    } slow;
  };
  alignas(8) uint32_t coarse[COARSE];
  u64 key[LIST];
  uint16_t group[LIST];
  double table[TABLE];               // for the weights
  u64 warp[WARPS];
  double warp_d[WARPS];
  float max[WARPS], part_max;
  int n_key, n_group, first_bin, last_bin;
  u64 found, before, total, certain, count_before, sum_of_all;
  uint32_t low_order, high_order, base, top;
  int mode, shift;
  Request request;
};

constexpr u64 NOTHING = 0x4330000000000000ull;      // 2^52 as a double

// A row's weights 2^t, t = (x - m) c log2(e) <= 0, in 64 bits and as whole numbers, exact to 2e-14 of themselves.  One fused multiply-add
// gives t as a whole number of 2^-45, in the lower bits of a double of the size of 1.5 2^52: t = n + i/16 + g/16.  2^(i/16) comes from a table
// of as many numbers as shared memory has 64-bit banks, 2^(g/16) from a polynomial in z = 1 + g that meets it at six Chebyshev points of
// [1, 2) (5e-15), and n is added to the table's exponent.  64-bit operations, seven of them, bound the passes that weigh every token:
// with nothing else in the loop a multiprocessor takes 7.6 cycles for 32 tokens, 2.4 of them for the conversion and the first operation.  A table of 256 saves one and costs as much in bank conflicts.  Rounding
// m c log2(e) to 2^-33 (a common factor of all weights) asks for |m c log2(e)| < 2^20.
constexpr double MAGIC = 6755399441055744.0;         // 1.5 2^52
__device__ __forceinline__ u64 raw_weight(float x, double C, double K, float low, const double* table) {
  const double r = fma(double(fmaxf(x, low)), C, K);
  const uint32_t hi = uint32_t(__double2hiint(r)), lo = uint32_t(__double2loint(r));
  const double z = __hiloint2double(int((__funnelshift_r(lo, hi, 21) & 0xfffffu) | 0x3ff00000u), int(lo << 11)), e = table[(hi >> 9) & (TABLE - 1)];
  const double p = fma(fma(fma(fma(fma(1.299453103455795e-09, z, 1.402322708390649e-07), z, 1.2976900509924959e-05), z, 0.0008985996992888076), z, 0.04148500125886912), z, 0.9576032806096036);
  return u64(__double_as_longlong(fma(p, __hiloint2double(__double2hiint(e) + int((hi << 7) & 0xfff00000u), __double2loint(e)), 4503599627370496.0)));
}
struct Weights {
  double m, c2, unit, C, K;
  float low;                         // a weight of 2^-60, which is nothing
  const double* table;
  __device__ __forceinline__ Weights(float largest, float scale, double unit, const double* table)
      : m(largest), c2(double(scale) * 1.4426950408889634), unit(unit), C(c2 * 0x1p45), K(MAGIC - m * C), low(float(m - 60.0 / c2)), table(table) {}
  __device__ __forceinline__ bool extreme() const { return !(fabs(m * c2) < 1048576.0) || !(low > -3.0e38f); }
  // Number i of the table, its exponent such that what stands above the fraction of t only has to be added.
  __device__ static double entry(int i, double unit) {
    const double e = exp2(double(i) / TABLE) * unit;
    return __hiloint2double(int(uint32_t(__double2hiint(e)) - 0x9C000000u), __double2loint(e));
  }
  __device__ __forceinline__ u64 raw(float x) const { return raw_weight(x, C, K, low, table); }      // NOTHING and the whole number
  __device__ __forceinline__ u64 whole(float x) const { return raw(x) - NOTHING; }
  __device__ __forceinline__ double log_factor() const { return (fma(m, C, K) - MAGIC) * (0x1p-45 * 0.6931471805599453); }      // of the common factor
  __device__ __forceinline__ u64 any(float x) const { return u64(exp2((double(x) - m) * c2) * unit + 0.5); }      // of extreme rows
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

// The sum of v over the threads before this one, and over all of them.
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
__device__ __forceinline__ double scan_before(double v, Smem& s, double& all) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  double incl = v;
  for (int o = 1; o < 32; o <<= 1) {
    const double y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();
  if (lane == 31) s.warp_d[w] = incl;
  __syncthreads();
  double at = incl - v;
  all = 0.0;
  for (int i = 0; i < WARPS; ++i) {
    at += i < w ? s.warp_d[i] : 0.0;
    all += s.warp_d[i];
  }
  return at;
}

// Sorts n keys in descending order.  A key for each thread: by counting the larger ones (256: 1 us).  More: in a network, in which pairs up to
// 32 apart belong to one warp, and the keys behind them, up to a power of two, are overwritten (1024: 5 us).
__device__ __noinline__ void sort_keys(u64* key, int n) {
  if (n <= TPB) {
    __syncthreads();
    u64 mine = 0;
    int place = 0;
    if (int(threadIdx.x) < n) {
      mine = key[threadIdx.x];
#pragma unroll 8
      for (int j = 0; j < n; ++j) place += key[j] > mine;
    }
    __syncthreads();
    if (int(threadIdx.x) < n) key[place] = mine;
    __syncthreads();
    return;
  }
  int size = 64;
  while (size < n) size *= 2;
  for (int i = n + threadIdx.x; i < size; i += TPB) key[i] = 0;
  __syncthreads();
#pragma unroll 1
  for (int k = 2; k <= size; k *= 2)
#pragma unroll 1
    for (int j = k / 2; j; j /= 2) {
      for (int p = threadIdx.x; p < size / 2; p += TPB) {
        const int i = 2 * p - (p & (j - 1));
        const u64 a = key[i], b = key[i + j];
        if (((i & k) == 0) == (a < b)) {
          key[i] = b;
          key[i + j] = a;
        }
      }
      if (j > 32 || (j == 1 && k >= 64)) __syncthreads();
      else __syncwarp();
    }
  __syncthreads();
}

// The smallest whole number not below p all, p in (0, 1), exactly, and at least 1.
__device__ __forceinline__ u64 start_of(float p, u64 all) {
  const uint32_t b = __float_as_uint(p);
  const int e = int(b >> 23), down = 150 - (e ? e : 1);
  const u64 f = (b & 0x7fffffu) | (e ? 0x800000u : 0u), lo = f * all, hi = __umul64hi(f, all), n = share_of(p, all);
  const bool whole = down < 64 ? (lo & ((1ull << down) - 1)) == 0 : down < 128 && lo == 0 && (hi & ((1ull << (down - 64)) - 1)) == 0;
  return max(u64(1), n + (whole ? 0 : 1));
}

__device__ __forceinline__ Request request_of(const SampleArgs& a, int64_t t) {
  Request q;
  q.u = a.u[t];
  q.scale = a.scale ? a.scale[t] : 1.0f;
  q.p = a.top_p ? a.top_p[t] : 1.0f;
  q.mp = a.min_p ? a.min_p[t] : 0.0f;
  q.k = a.top_k ? a.top_k[t] : 0;
  q.valid = q.scale > 0.0f && q.scale < INFINITY && !isnan(q.p) && !isnan(q.mp) && !isnan(q.u);
  if (q.p <= 0.0f || q.mp > 1.0f) q.k = 1;
  q.mp = fminf(q.mp, 1.0f);
  if (q.k <= 0 || q.k > a.V) q.k = a.V;
  if (q.k == 1) q.p = 1.0f;
  return q;
}

__device__ __forceinline__ void put_token(const SampleArgs& a, int64_t t, int64_t token, float logprob) {
  if (a.id_type == MV_I32) static_cast<int32_t*>(a.token)[t] = int32_t(token);
  else static_cast<int64_t*>(a.token)[t] = token;
  if (a.logprob) a.logprob[t] = logprob;
}
// The log of a token's share: of one half and more by what is missing to one, a whole number (0 where nothing is), of less by its logit,
// since a light weight is a rounded one.
__device__ __forceinline__ void put_drawn(const SampleArgs& a, int64_t t, int64_t token, float x, const Weights& wt, u64 weight, u64 all, double log_factor) {
  const u64 rest = all - weight;
  const double share = rest < weight ? 0.0 - log1p(double(rest) / double(weight))
                                     : (double(x) - wt.m) * (wt.c2 * 0.6931471805599453) - log(double(all) / wt.unit) + log_factor;
  put_token(a, t, token, float(share));
}
__device__ __forceinline__ u64 limit_of(float u, u64 all) { return u >= 1.0f ? all - 1 : u > 0.0f ? share_of(u, all) : 0; }      // the first token at which the sum is larger is drawn

// The smallest logit for which f holds, f false below it and true from it on; +inf: none.  By all lanes of a warp, five bits of the
// order at a time.
template <typename F> __device__ __forceinline__ float smallest(F&& f) {
  const uint32_t lane = threadIdx.x & 31;
  constexpr uint32_t LOW = 0x00800000u, HIGH = 0xff7fffffu;          // the orders of the finite numbers
  uint32_t base = 0;                 // f is false below it
  for (int shift = 27; ; shift = shift > 5 ? shift - 5 : 0) {
    const uint32_t h = base + (lane << shift);
    const bool over = h < base;      // past 2^32
    const unsigned hit = __ballot_sync(0xffffffffu, over || h > HIGH || (h >= LOW && f(value_of(h))));
    const int n = hit ? __ffs(int(hit)) - 1 : 32;      // the first place where it holds
    if (shift == 0) {
      base += uint32_t(n);
      break;
    }
    base += n ? uint32_t(n - 1) << shift : 0;
  }
  return base > HIGH ? INFINITY : value_of(base);
}

// ------------------------------------------------------------------------------------------ any row
// Rows that the fast paths do not take: cuts by three readings each, over 11, 11 and 10 bits of the order.
struct Cut { uint32_t order; int64_t ties, all; };       // kept: larger orders, and the first `ties` of the `all` tokens of this order

// Cuts the tokens that `floor` keeps (all of them: null) to the shortest start, in descending order, that holds at least `target` (> 0)
// of what `amount` gives to each; there is one.
template <typename X, typename F>
__device__ __noinline__ Cut cut_row(const X* row, int64_t V, u64 target, const Cut* floor, F&& amount, Smem& s) {
  uint32_t prefix = 0;
  u64 before = 0;
  int shift = 32;
  for (int step = 0; step < 3; ++step) {
    const int bits = step < 2 ? 11 : 10, next = shift - bits;
    __syncthreads();
    for (int i = threadIdx.x; i < SLOW_BINS; i += TPB) s.slow.bin[i] = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < V; i += TPB) {
      const float x = to_f(row[i]);
      const uint32_t h = order_of(x);
      if ((shift == 32 || h >> shift == prefix) && (!floor || h >= floor->order)) {
        const u64 v = amount(x);
        if (v) atomicAdd(&s.slow.bin[(h >> next) & ((1u << bits) - 1)], v);
      }
    }
    __syncthreads();
    if (floor && threadIdx.x == 0 && (shift == 32 || floor->order >> shift == prefix))   // the tokens of the floor's own order that it drops
      s.slow.bin[(floor->order >> next) & ((1u << bits) - 1)] -= amount(value_of(floor->order)) * u64(floor->all - floor->ties);
    __syncthreads();
    // bins in descending order, eight per thread
    constexpr int PER = SLOW_BINS / TPB;
    u64 mine = 0, all;
    for (int j = 0; j < PER; ++j) mine += s.slow.bin[SLOW_BINS - 1 - (threadIdx.x * PER + j)];
    u64 at = before + scan_before(mine, s, all);
    for (int j = 0; j < PER; ++j) {
      const int b = SLOW_BINS - 1 - (threadIdx.x * PER + j);
      if (at < target && target <= at + s.slow.bin[b]) {
        s.first_bin = b;
        s.before = at;
      }
      at += s.slow.bin[b];
    }
    __syncthreads();
    prefix = prefix << bits | uint32_t(s.first_bin);
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
__device__ __noinline__ void sample_any(const X* row, const SampleArgs& a, int64_t t, const Request& q, const Weights& wt, Smem& s) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const bool extreme = wt.extreme();
  // the fast paths' weights to the bit, so that a row's token does not hang on the path that it takes
  auto weight = [&](float x) { return extreme ? wt.any(x) : wt.whole(x); };
  Cut cut = {0, 0, 0};               // all
  bool cuts = false;
  if (q.k < a.V) {
    cut = cut_row(row, a.V, u64(q.k), nullptr, [](float) { return u64(1); }, s);
    cuts = true;
  }
  if (q.p < 1.0f) {
    u64 mine = 0, all;
    for (int64_t i = threadIdx.x; i < a.V; i += TPB) {
      const float x = to_f(row[i]);
      if (!cuts || order_of(x) > cut.order) mine += weight(x);
    }
    scan_before(mine, s, all);
    if (cuts) all += u64(cut.ties) * weight(value_of(cut.order));
    const u64 target = start_of(q.p, all);
    cut = cut_row(row, a.V, target, cuts ? &cut : nullptr, weight, s);
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
      if (tie && at + 1 == u64(cut.ties)) s.found = u64(i);
      found += all;
      if (found >= u64(cut.ties)) break;
    }
    __syncthreads();
    last = int64_t(s.found);
  }
  auto kept = [&](int64_t i) {       // the weight of token i, 0 if it is cut
    const float x = to_f(row[i]);
    const uint32_t h = order_of(x);
    if (cuts && !(h > cut.order || (h == cut.order && i <= last))) return u64(0);
    return exp((double(x) - wt.m) * double(q.scale)) >= double(q.mp) ? weight(x) : u64(0);
  };
  const int64_t per = ((a.V + CHUNKS - 1) / CHUNKS + 31) / 32 * 32;
  __syncthreads();
  for (int c = w; c < CHUNKS; c += WARPS) {
    u64 n = 0;
    for (int64_t i = c * per + lane; i < min(a.V, (c + 1) * per); i += 32) n += kept(i);
    for (int o = 16; o; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    if (lane == 0) s.slow.chunk[c] = n;
  }
  __syncthreads();
  constexpr int PER = CHUNKS / TPB;
  u64 mine = 0, all;
  for (int j = 0; j < PER; ++j) mine += s.slow.chunk[threadIdx.x * PER + j];
  u64 at = scan_before(mine, s, all);
  const u64 limit = limit_of(q.u, all);
  for (int j = 0; j < PER; ++j) {
    const u64 n = s.slow.chunk[threadIdx.x * PER + j];
    if (at <= limit && limit < at + n) {
      s.first_bin = threadIdx.x * PER + j;
      s.before = at;
    }
    at += n;
  }
  __syncthreads();
  if (w) return;
  u64 before = s.before;
  for (int64_t i0 = int64_t(s.first_bin) * per; i0 < a.V; i0 += 32) {
    const int64_t i = i0 + lane;
    const u64 n = i < a.V ? kept(i) : 0;
    u64 incl = n;
    for (int o = 1; o < 32; o <<= 1) {
      const u64 y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, before + incl > limit);
    if (hit) {
      if (lane == __ffs(int(hit)) - 1) put_drawn(a, t, i, to_f(row[i]), wt, n, all, extreme ? 0.0 : wt.log_factor());
      return;
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
}

// ------------------------------------------------------------------------------------------ fast paths
template <typename X> __device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t max2_nan<float>(uint32_t a, uint32_t b) { return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b))); }
template <> __device__ __forceinline__ uint32_t max2_nan<__nv_bfloat16>(uint32_t a, uint32_t b) { return Vec<__nv_bfloat16>::max2_nan(a, b); }
template <> __device__ __forceinline__ uint32_t max2_nan<__half>(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <typename X> __device__ __forceinline__ float widen_nan(uint32_t m) {
  if constexpr (sizeof(X) == 4) {
    return __uint_as_float(m);
  } else {
    float a, b;
    unpack2(Vec<X>::pair(make_uint4(m, 0, 0, 0), 0), a, b);
    return max_nan(a, b);
  }
}

// f(chunk of the CTA's, a lane's vectors of it), the next ones on their way; what is not of the row is masked.
template <typename X, typename F> __device__ __forceinline__ void walk(const uint4* vec, int nv, F&& f) {
  constexpr int OWN = CHUNK / Vec<X>::N / 32;
  const int tid = threadIdx.x, turns = (nv + OWN * TPB - 1) / (OWN * TPB);
  uint4 u[OWN], next[OWN];
  auto fetch = [&](int i) {
#pragma unroll
    for (int j = 0; j < OWN; j += 2) {
      next[j] = next[j + 1] = make_uint4(Vec<X>::NONE, Vec<X>::NONE, Vec<X>::NONE, Vec<X>::NONE);
      if ((i * TPB + tid) * OWN + j < nv) load_stream(vec + (i * TPB + tid) * OWN + j, next[j], next[j + 1]);
    }
  };
  fetch(0);
#pragma unroll 1
  for (int i = 0; i < turns; ++i) {
#pragma unroll
    for (int j = 0; j < OWN; ++j) u[j] = next[j];
    fetch(i + 1);
    f(i * WARPS + (tid >> 5), u);
  }
}

// What happens to a logit between the thresholds.
enum { LISTED, BINNED, TIED };
__device__ __forceinline__ void push(Smem& s, float x, int col) {
  const int i = atomicAdd(&s.n_key, 1);
  if (i < LIST) s.key[i] = make_key(x, uint32_t(col));
}
__device__ __forceinline__ void note(Smem& s, float x, int col) {
  if (s.mode == LISTED) {
    push(s, x, col);
  } else if (s.mode == BINNED) {
    atomicAdd(&s.fast.bin[(order_of(x) - s.base) >> s.shift], 1u);
  } else {
    atomicMin(&s.low_order, order_of(x));
    atomicMax(&s.high_order, order_of(x));
  }
}

// The weights of a CTA's vectors (from column col0 of the row on): their sums by chunks, of the logits from t1 on; those in [t2, t1) are noted.
// KIND 0: of all; 1: of those from t2 on; 2: of all, with the sum of all, of which a thread's part is returned.  A function of its own, so
// that it has all of the registers.
template <typename X, int KIND>
__device__ __noinline__ u64 weigh(const X* row, int col0, int nv, double C, double K, float low, float t1, float t2) {
  constexpr int N = Vec<X>::N, CHUNK_VECS = CHUNK / N, OWN = CHUNK_VECS / 32;
  extern __shared__ u64 dynamic[];
  Smem& s = *reinterpret_cast<Smem*>(dynamic);
  const int lane = threadIdx.x & 31;
  u64 total = 0;
  walk<X>(reinterpret_cast<const uint4*>(row + col0), nv, [&](int chunk, const uint4 (&u)[OWN]) {
    u64 v = 0;
    unsigned hit = 0;
#pragma unroll
    for (int i = 0; i < OWN; ++i)
      each_logit<X>(u[i], [&](int e, float y) {
        if (KIND == 1 && !__any_sync(0xffffffffu, y >= t2)) return;            // few of them
        const u64 weight = raw_weight(y, C, K, low, s.table) - NOTHING;
        if (KIND == 2) total += weight;
        v += KIND == 0 || y >= t1 ? weight : 0;
        if (KIND) hit |= y >= t2 && y < t1 ? 1u << (i * N + e) : 0u;
      });
    if (KIND == 1 && s.mode == TIED) {
      const unsigned ties = __reduce_add_sync(0xffffffffu, unsigned(__popc(hit)));
      if (lane == 0 && chunk * CHUNK_VECS < nv) s.fast.bin[1 + chunk] = ties;
    }
    for (; hit; hit &= hit - 1) {
      const int col = col0 + chunk * CHUNK + 16 * lane + __ffs(int(hit)) - 1;
      note(s, to_f(row[col]), col);
    }
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0 && chunk * CHUNK_VECS < nv) s.fast.chunk[1 + chunk] = v;
  });
  return total;
}

// The bin of a logit among `n`: 0 at the largest one, the last one for all that is 2^-32 of its weight or less.  Never falls as x falls.
__device__ __forceinline__ int bin_of(float x, float m, float c, int n) { return int(fminf(distance(m, x, c), float(n - 1))); }

template <typename X>
__global__ void __launch_bounds__(TPB, RESIDENT) k_sample(const X* __restrict__ logits, const __grid_constant__ SampleArgs a) {
  constexpr int N = Vec<X>::N, CHUNK_VECS = CHUNK / N, OWN = CHUNK_VECS / 32;      // OWN: vectors of a chunk that a lane has
  extern __shared__ u64 dynamic[];
  Smem& s = *reinterpret_cast<Smem*>(dynamic);
  const cg::cluster_group cluster = cg::this_cluster();
  const int ctas = int(cluster.num_blocks()), rank = int(cluster.block_rank());
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int64_t t = ctas == 1 ? blockIdx.x : blockIdx.x / unsigned(ctas);
  const X* row = logits + t * a.ld;
  const Request q = request_of(a, t);
  // the vectors begin at the row's first 32-byte boundary; `per` of them for each CTA of the cluster
  const int64_t to32 = int64_t((32 - (reinterpret_cast<uintptr_t>(row) & 31)) & 31) / int(sizeof(X));
  const int first = int(min(a.V, to32)), all_v = (int(a.V) - first) / (2 * N) * 2;
  const int per = ((all_v + ctas - 1) / ctas + CHUNK_VECS - 1) / CHUNK_VECS * CHUNK_VECS, v0 = min(all_v, rank * per), nv = min(all_v - v0, per);
  const int tail_col = first + all_v * N, head = rank == 0 ? first : 0, tail = rank == ctas - 1 ? int(a.V) - tail_col : 0;
  const uint4* vec = reinterpret_cast<const uint4*>(row + first) + v0;
  const int col0 = first + v0 * N;
  const int end_col = tid < head ? tid : tid - head < tail ? tail_col + tid - head : -1;      // a single logit of this thread
  const float end = end_col >= 0 ? to_f(row[end_col]) : -INFINITY;
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
  auto stream = [&](auto&& f) {      // f(step, vectors), the next step's on their way
    uint4 even[U], odd[U];
    if (n_steps > 0) load(0, even);
    for (int step = 0; step < n_steps; step += 2) {
      if (step + 1 < n_steps) load(step + 1, odd);
      f(step, even);
      if (step + 1 >= n_steps) break;
      if (step + 2 < n_steps) load(step + 2, even);
      f(step + 1, odd);
    }
  };
  auto all_sync = [&]() {
    if (ctas > 1) cluster.sync();
    else __syncthreads();
  };
  auto of_rank = [&](int r) -> const Smem& { return ctas > 1 ? *cluster.map_shared_rank(&s, unsigned(r)) : s; };
  if (tid < TABLE) s.table[tid] = Weights::entry(tid, a.unit);

  // the largest logit, and those of the groups where the top k are asked for
  bool by_list = q.k <= LIST && q.k < a.V;
  float m = end;
  {
    float g = -INFINITY;
    int left = a.steps, group = 0;
    stream([&](int, const uint4 (&u)[U]) {
      uint32_t m2 = max2_nan<X>(max2_nan<X>(u[0].x, u[0].y), max2_nan<X>(u[0].z, u[0].w));
#pragma unroll
      for (int i = 1; i < U; ++i) m2 = max2_nan<X>(m2, max2_nan<X>(max2_nan<X>(u[i].x, u[i].y), max2_nan<X>(u[i].z, u[i].w)));
      const float v = widen_nan<X>(m2);
      m = max_nan(m, v);
      if (by_list) {
        g = max_nan(g, v);
        if (--left == 0) {
          s.gmax[group++][tid] = g;
          g = -INFINITY;
          left = a.steps;
        }
      }
    });
    if (by_list && left != a.steps) s.gmax[group][tid] = g;
  }
  const int groups = (n_steps + a.steps - 1) / a.steps;
  for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) s.max[w] = m;
  for (int i = tid; i < COARSE; i += TPB) s.coarse[i] = 0;
  if (tid == 0) {
    s.n_key = s.n_group = 0;
    s.low_order = 0xffffffffu;
    s.high_order = 0;
    s.request = q;
  }
  __syncthreads();
  for (int i = 0; i < WARPS; ++i) m = max_nan(m, s.max[i]);
  if (ctas > 1) {
    if (tid == 0) s.part_max = m;
    cluster.sync();
    m = max_nan(m, of_rank(lane % ctas).part_max);
    for (int o = 4; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));      // at most eight
  }
  if (!(m < INFINITY) || !q.valid || m == -INFINITY) {
    if (ctas > 1) cluster.sync();    // the parts' maxima have been read
    if (rank == 0 && tid == 0) put_token(a, t, -1, q.valid && m == -INFINITY ? -INFINITY : NAN);
    return;
  }
  const Weights wt(m, q.scale, a.unit, s.table);
  const bool extreme = wt.extreme();
  by_list &= !extreme;
  const float c_coarse = fminf(q.scale * (LOG2E * 16.0f), 3.0e38f), c_fine = fminf(q.scale * (LOG2E * 128.0f), 3.0e38f);
  const float t_mp = q.mp <= 0.0f ? -INFINITY : smallest([&](float x) { return exp((double(x) - wt.m) * double(q.scale)) >= double(q.mp); });      // min p as a logit

  // the other CTAs' lists behind the first one's, a warp for each; own: the length of the list of CTA `lane`
  auto gather = [&](int own) {
    int base = own;
    for (int o = 1; o < MOST_CTAS; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, base, o);
      if (lane >= o) base += y;
    }
    const int from = __shfl_sync(0xffffffffu, base - own, w), more = __shfl_sync(0xffffffffu, own, w);
    if (w && w < ctas)
      for (int i = lane; i < more; i += 32) s.key[from + i] = of_rank(w).key[i];
  };

  if (by_list) {
    // the coarse bin up to which k of what the CTAs have counted lie (COARSE: none), and how much they have counted
    u64 counted;
    auto bin_of_k = [&]() {
      all_sync();
      u64 c[2] = {0, 0};
#pragma unroll
      for (int r = 0; r < MOST_CTAS; ++r) {
        const uint2 v = r < ctas ? *reinterpret_cast<const uint2*>(&of_rank(r).coarse[2 * tid]) : make_uint2(0, 0);
        c[0] += v.x;
        c[1] += v.y;
      }
      if (tid == 0) s.first_bin = COARSE;
      const u64 at = scan_before(c[0] + c[1], s, counted);
      if (at < u64(q.k) && u64(q.k) <= at + c[0] + c[1]) s.first_bin = 2 * tid + (at + c[0] < u64(q.k));
      __syncthreads();
      return s.first_bin;
    };
    // k groups' maxima lie up to bin b: so do k logits, and all of the top k
    for (int g = 0; g < groups; ++g) atomicAdd(&s.coarse[bin_of(s.gmax[g][tid], m, c_coarse, COARSE)], 1u);
    if (end_col >= 0) atomicAdd(&s.coarse[bin_of(end, m, c_coarse, COARSE)], 1u);
    int b = bin_of_k();
    if (b >= COARSE - 1) {
      // too few groups (a short row, or one that is masked but for a few tokens): the logits are counted, those of the last bin, which has the
      // masked ones too, by each thread (2 rows of 3200 f16, 97 % masked, k 50, p 0.9: 78 us without this)
      all_sync();
      for (int i = tid; i < COARSE; i += TPB) s.coarse[i] = 0;
      __syncthreads();
      uint32_t last = 0;
      auto count = [&](float y) {
        const int i = bin_of(y, m, c_coarse, COARSE);
        if (i < COARSE - 1) atomicAdd(&s.coarse[i], 1u);
        else last += y > -INFINITY;
      };
#pragma unroll 2
      for (int v = tid; v < nv; v += TPB) each_logit<X>(__ldg(vec + v), [&](int, float y) { count(y); });
      if (end_col >= 0) count(end);
      last = __reduce_add_sync(0xffffffffu, last);
      if (lane == 0 && last) atomicAdd(&s.coarse[COARSE - 1], last);
      b = min(bin_of_k(), COARSE - 1);
      by_list = b < COARSE - 1 || counted <= LIST;
    }
    if (q.p >= 1.0f && q.mp > 0.0f) b = min(b, bin_of(t_mp, m, c_coarse, COARSE));      // nothing beyond it is kept
    if (by_list) {
      for (int g = 0; g < groups; ++g)
        if (s.gmax[g][tid] > -INFINITY && bin_of(s.gmax[g][tid], m, c_coarse, COARSE) <= b) {
          const int i = atomicAdd(&s.n_group, 1);
          if (i < LIST) s.group[i] = uint16_t(g * TPB + tid);
        }
      if (end > -INFINITY && bin_of(end, m, c_coarse, COARSE) <= b) push(s, end, end_col);
      __syncthreads();
      const int listed = s.n_group, vecs = a.steps * U;
      if (listed <= LIST) {
        for (int i = tid; i < listed * vecs; i += TPB) {
          const int g = s.group[i / vecs], j = i % vecs, v = (g / TPB * vecs + (j & ~1)) * TPB + 2 * (g % TPB) + (j & 1);
          if (v >= nv) continue;
          const uint4 x = __ldg(vec + v);
          each_logit<X>(x, [&](int e, float y) {
            if (y > -INFINITY && bin_of(y, m, c_coarse, COARSE) <= b) push(s, y, col0 + v * N + e);
          });
        }
      } else if (tid == 0) {
        s.n_key = LIST + 1;
      }
    }
    all_sync();
    const int own = lane < ctas ? min(of_rank(lane).n_key, LIST + 1) : 0, n = __reduce_add_sync(0xffffffffu, own);
    by_list = by_list && n <= LIST;
    if (by_list) {
      if (rank == 0) gather(own);
      all_sync();
      if (rank) return;
      // sorted, summed up in descending order, cut, summed up by index
      sort_keys(s.key, n);
      constexpr int PER = LIST / TPB;
      u64 v[PER], mine = 0, total;
      const int kept_k = int(min(q.k, int64_t(n)));
      for (int j = 0; j < PER; ++j) {
        const int i = tid * PER + j;
        v[j] = i < kept_k ? wt.whole(key_value(s.key[i])) : 0;
        mine += v[j];
      }
      u64 before = scan_before(mine, s, total);
      const u64 target = q.p < 1.0f ? start_of(q.p, total) : ~0ull;
      for (int j = 0; j < PER; ++j) {
        const int i = tid * PER + j;
        const bool in = i < kept_k && (i == 0 || (before < target && key_value(s.key[i]) >= t_mp));
        before += v[j];
        if (!in) v[j] = 0;
        if (i < n) {
          s.fast.sum[i] = v[j];
          s.fast.sorted[i] = u64(uint32_t(s.key[i])) << 32 | unsigned(i);       // by index, and the place among the keys
        }
      }
      sort_keys(s.fast.sorted, n);
      mine = 0;
      for (int j = 0; j < PER; ++j) {
        const int i = tid * PER + j;
        v[j] = i < n ? s.fast.sum[uint32_t(s.fast.sorted[i])] : 0;
        mine += v[j];
      }
      before = scan_before(mine, s, total);
      const u64 limit = limit_of(q.u, total);
      for (int j = 0; j < PER; ++j) {
        if (before <= limit && limit < before + v[j]) {
          const u64 key = s.key[uint32_t(s.fast.sorted[tid * PER + j])];
          put_drawn(a, t, key_index(key), key_value(key), wt, v[j], total, wt.log_factor());
        }
        before += v[j];
      }
      return;
    }
    all_sync();                      // the lists' lengths have been read
    if (tid == 0) s.n_key = 0;
  }

  // The sums of all CTAs' bins (which are complete) in each of them; neighbouring threads take neighbouring bins.
  auto sum_bins = [&]() {
    if (ctas == 1) return;
    uint32_t c[FINE / TPB] = {};
#pragma unroll 2
    for (int r = 0; r < ctas; ++r) {
      const Smem& o = of_rank((rank + r) % ctas);
#pragma unroll
      for (int j = 0; j < FINE / TPB; ++j) c[j] += o.fast.bin[j * TPB + tid];
    }
    all_sync();
#pragma unroll
    for (int j = 0; j < FINE / TPB; ++j) s.fast.bin[j * TPB + tid] = c[j];
    __syncthreads();
  };
  auto clear_bins = [&]() {
    __syncthreads();
    for (int i = tid; i < FINE; i += TPB) s.fast.bin[i] = 0;
    __syncthreads();
  };

  // bins of all logits, where a cut is asked for: the bins [lo, hi] in which the last token of the start may lie, and their logits [t2, t1)
  float t1 = -INFINITY, t2 = -INFINITY;
  bool slow = a.chunks == 0 || extreme, cut = false, crowd = false;      // crowd: more than the list holds
  const bool by_count = q.k < a.V, by_mass = q.p < 1.0f;
  u64 count_before = 0;
  if (by_count && by_mass) slow = true;
  if (!slow && (by_count || by_mass)) {
    clear_bins();
    if (end > -INFINITY) atomicAdd(&s.fast.bin[bin_of(end, m, c_fine, FINE)], 1u);
    walk<X>(vec, nv, [&](int, const uint4 (&u)[OWN]) {
#pragma unroll
      for (int i = 0; i < OWN; ++i)
        each_logit<X>(u[i], [&](int, float y) {
          if (y > -INFINITY) atomicAdd(&s.fast.bin[bin_of(y, m, c_fine, FINE)], 1u);
        });
    });
    all_sync();
    constexpr int PER = FINE / TPB;
    sum_bins();
    uint32_t c[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) c[j] = s.fast.bin[tid * PER + j];
    if (tid == 0) { s.first_bin = s.last_bin = FINE - 1; s.before = 0; }
    bool enough = false;
    if (by_count) {
      u64 mine = 0, all;
      for (int j = 0; j < PER; ++j) mine += c[j];
      u64 at = scan_before(mine, s, all);
      enough = all < u64(q.k);       // masks leave fewer
      for (int j = 0; j < PER; ++j) {
        if (at < u64(q.k) && u64(q.k) <= at + c[j]) {
          s.first_bin = s.last_bin = tid * PER + j;
          s.before = at;
        }
        at += c[j];
      }
    } else {
      // A bin's weights lie within 2^(-1/128) of one another; what 32 bits round is a hundredth of the slack.  The start ends in the first bin
      // at whose end (1 - p) times the sum up to it is no less than p times the rest.
      const double step = exp2(-1.0 / 128.0), low = step * (1.0 - 2e-4), top = exp2(-double(tid * PER) / 128.0) * (1.0 + 1e-4), p = double(q.p);
      double most = 0.0, all_most, all_least, v = top;
      for (int j = 0; j < PER; ++j, v *= step) most += c[j] * v;
      double last = tid == TPB - 1 ? c[PER - 1] * exp2(-double(FINE - 1) / 128.0) * (1.0 + 1e-4) : 0.0;      // the last bin's may be nothing
      double at_most = scan_before(most, s, all_most), at_least = scan_before((most - last) * low, s, all_least);
      v = top;
      // Two threads may each see their first one at their border, where the scan and the running sum round differently: the lower one counts, in
      // every CTA of the cluster alike.
      unsigned lo_at = FINE - 1, hi_at = FINE - 1;
      for (int j = 0; j < PER; ++j, v *= step) {
        at_most += c[j] * v;
        at_least += c[j] * v * low;
        if ((1.0 - p) * at_most >= p * (all_least - at_least)) lo_at = min(lo_at, unsigned(tid * PER + j));
        if ((1.0 - p) * at_least >= p * (all_most - at_most)) hi_at = min(hi_at, unsigned(tid * PER + j));
      }
      lo_at = __reduce_min_sync(0xffffffffu, lo_at);
      hi_at = __reduce_min_sync(0xffffffffu, hi_at);
      if (lane == 0) {
        atomicMin(&s.first_bin, int(lo_at));
        atomicMin(&s.last_bin, int(hi_at));
      }
    }
    __syncthreads();
    const int lo = s.first_bin, hi = s.last_bin;
    count_before = s.before;
    u64 mine = 0, in_range;
    for (int j = 0; j < PER; ++j) mine += tid * PER + j >= lo && tid * PER + j <= hi ? c[j] : 0;
    scan_before(mine, s, in_range);
    crowd = in_range > LIST;
    slow = !enough && (hi >= FINE - 1 || lo > hi);
    if (!slow && !enough) {
      t1 = lo == 0 ? INFINITY : smallest([&](float x) { return bin_of(x, m, c_fine, FINE) < lo; });
      t2 = smallest([&](float x) { return bin_of(x, m, c_fine, FINE) <= hi; });
      cut = t_mp < t1;               // else min p leaves nothing of them
    }
  }
  if (slow) {
    all_sync();                      // what the others read of this CTA has been read
    if (rank == 0) sample_any<X>(row, a, t, q, wt, s);
    return;
  }

  crowd &= cut;
  if (!cut) t1 = t2 = t_mp;
  // Weights: sums of neighbours among the logits from t1 on, and, for a cut by mass, the sum of all.  What is in [t2, t1) is listed; where it is
  // a crowd (few distinct values, as 16 bits leave them), counted in bins by its order, which narrow [t2, t1), and in a second pass listed or,
  // where it is a crowd of one value, counted by chunks.
  // (What only the seldom parts need waits in shared memory: the passes' registers are few.)
  if (tid == 0) {
    s.mode = crowd ? BINNED : LISTED;
    s.count_before = count_before;
    if (crowd) {
      s.base = order_of(t2);
      s.top = t1 == INFINITY ? order_of(m) + 1 : order_of(t1);
      s.shift = 0;
      while ((s.top - 1 - s.base) >> s.shift >= FINE) ++s.shift;
    }
  }
  const int own_chunks = (nv + CHUNK_VECS - 1) / CHUNK_VECS, chunks = 2 + (all_v + CHUNK_VECS - 1) / CHUNK_VECS;
  auto sums = [&](auto kind) {
    constexpr int KIND = decltype(kind)::value;
    u64 total = weigh<X, KIND>(row, col0, nv, wt.C, wt.K, wt.low, t1, t2), all;
    // the ends: chunk 0 is the head, the one behind the last is the tail
    if (w == 0) {
      const u64 weight = wt.whole(end);
      u64 v = end >= t1 ? weight : 0, h = end_col >= 0 && end_col < first ? v : 0;
      v -= h;
      total += weight;
      if (end >= t2 && end < t1) {
        note(s, end, end_col);
        if (s.mode == TIED) atomicAdd(&s.fast.bin[end_col < first ? 0 : 1 + own_chunks], 1u);
      }
      for (int o = 16; o; o >>= 1) {
        v += __shfl_xor_sync(0xffffffffu, v, o);
        h += __shfl_xor_sync(0xffffffffu, h, o);
      }
      if (lane == 0) {
        if (rank == 0) s.fast.chunk[0] = h;
        if (rank == ctas - 1) s.fast.chunk[1 + own_chunks] = v;
      }
    }
    scan_before(total, s, all);
    if (tid == 0) s.total = all;
  };
  // a number of every CTA, added up
  auto over_ctas = [&](u64 Smem::*field) {
    u64 v = lane < ctas ? of_rank(lane).*field : 0;
    for (int o = MOST_CTAS / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return __shfl_sync(0xffffffffu, v, 0);
  };
  if (crowd) clear_bins();
  for (;;) {
    __syncthreads();
    if (cut && by_mass && (!crowd || s.mode == BINNED)) sums(Int<2>());
    else if (t2 > -INFINITY) sums(Int<1>());
    else sums(Int<0>());
    if (s.mode != BINNED) break;
    u64 certain = 0;
    for (int i = (rank == 0 ? 0 : 1) + tid; i < 1 + own_chunks + (rank == ctas - 1); i += TPB) certain += s.fast.chunk[i];
    scan_before(certain, s, certain);
    if (tid == 0) s.certain = certain;
    all_sync();
    const u64 sum_of_all = over_ctas(&Smem::total);
    certain = by_count ? s.count_before : over_ctas(&Smem::certain);
    const u64 target = by_count ? u64(s.request.k) : start_of(s.request.p, sum_of_all);
    const uint32_t base = s.base, top = s.top;
    const int shift = s.shift;
    sum_bins();
    // In descending order: the place p is bin FINE - 1 - p.  The start ends between the first place whose bins, taken at their largest weights,
    // reach the target, and the first that does so at their smallest.
    constexpr int PER = FINE / TPB;
    auto weight = [&](uint32_t order) { return by_count ? u64(1) : wt.whole(value_of(order)); };
    u64 most = 0, least = 0, all;
    for (int j = 0; j < PER; ++j) {
      const uint32_t i = FINE - 1 - (tid * PER + j), n = s.fast.bin[i];
      if (n) {
        most += n * weight(min(top - 1, base + ((i + 1) << shift) - 1));
        least += n * weight(base + (i << shift));
      }
    }
    if (tid == 0) { s.first_bin = -1; s.last_bin = FINE - 1; s.before = 0; }
    u64 at_most = certain + scan_before(most, s, all), at_least = certain + scan_before(least, s, all);
    for (int j = 0; j < PER; ++j) {
      const uint32_t i = FINE - 1 - (tid * PER + j), n = s.fast.bin[i];
      if (n == 0) continue;
      most = n * weight(min(top - 1, base + ((i + 1) << shift) - 1));
      least = n * weight(base + (i << shift));
      if (at_most < target && target <= at_most + most) {
        s.first_bin = tid * PER + j;
        s.before = at_most;          // a cut by count: how many
      }
      if (at_least < target && target <= at_least + least) s.last_bin = tid * PER + j;
      at_most += most;
      at_least += least;
    }
    __syncthreads();
    const int lo = s.first_bin, hi = s.last_bin;
    u64 mine = 0;
    for (int j = 0; j < PER; ++j) mine += tid * PER + j >= lo && tid * PER + j <= hi ? s.fast.bin[FINE - 1 - (tid * PER + j)] : 0;
    scan_before(mine, s, all);
    if (lo < 0 || lo > hi) {         // never expected
      all_sync();
      if (rank == 0) sample_any<X>(row, a, t, s.request, wt, s);
      return;
    }
    const u64 edge = u64(base) + (u64(FINE - lo) << shift);          // above the place lo
    if (edge < top) t1 = value_of(uint32_t(edge));
    t2 = value_of(base + (uint32_t(FINE - 1 - hi) << shift));
    cut = t_mp < t1;
    if (!cut) t1 = t2 = t_mp;
    if (tid == 0) {
      s.mode = cut && all > LIST ? TIED : LISTED;
      s.count_before = s.before;
      s.sum_of_all = sum_of_all;
    }
    clear_bins();
  }
  all_sync();
  int n = 0;
  u64 sum_of_all = 0;
  uint32_t low_order = 0, high_order = 0;
  const int mode = s.mode;
  if (rank == 0) {
    const int own = lane < ctas ? min(of_rank(lane).n_key, LIST + 1) : 0;
    n = __reduce_add_sync(0xffffffffu, own);
    sum_of_all = crowd ? s.sum_of_all : over_ctas(&Smem::total);
    low_order = __reduce_min_sync(0xffffffffu, lane < ctas ? of_rank(lane).low_order : 0xffffffffu);
    high_order = __reduce_max_sync(0xffffffffu, lane < ctas ? of_rank(lane).high_order : 0);
    if (n <= LIST) gather(own);
    for (int i = tid; ctas > 1 && i < chunks; i += TPB) {
      const int r = min(ctas - 1, max(0, i - 1) / (per / CHUNK_VECS));
      if (r) {
        s.fast.chunk[i] = of_rank(r).fast.chunk[i - r * (per / CHUNK_VECS)];
        if (mode == TIED) s.fast.bin[i] = of_rank(r).fast.bin[i - r * (per / CHUNK_VECS)];
      }
    }
  }
  all_sync();
  if (rank) return;
  if (n > LIST || (mode == TIED && low_order != high_order)) {
    __syncthreads();
    sample_any<X>(row, a, t, s.request, wt, s);
    return;
  }
  auto bounds = [&](int c, int& from, int& to) {       // the columns of a chunk
    from = c == 0 ? 0 : c == chunks - 1 ? tail_col : first + (c - 1) * CHUNK;
    to = c == 0 ? first : c == chunks - 1 ? int(a.V) : min(tail_col, from + CHUNK);
  };
  constexpr int SHARE = CHUNK / TPB;                   // neighbouring tokens of a chunk per thread
  u64 last = 0;                      // the last kept token's key
  if (cut && mode == LISTED) {
    sort_keys(s.key, n);
    if (tid == 0) s.found = 0;
    __syncthreads();
    constexpr int PER = LIST / TPB;
    u64 v[PER], mine = 0, all, certain = 0;
    for (int i = tid; i < chunks; i += TPB) certain += s.fast.chunk[i];
    scan_before(certain, s, certain);
    for (int j = 0; j < PER; ++j) {
      const int i = tid * PER + j;
      v[j] = i >= n ? 0 : by_count ? 1 : wt.whole(key_value(s.key[i]));
      mine += v[j];
    }
    u64 at = (by_count ? s.count_before : certain) + scan_before(mine, s, all);
    const u64 target = by_count ? u64(s.request.k) : start_of(s.request.p, sum_of_all);
    for (int j = 0; j < PER; ++j) {
      if (at < target && target <= at + v[j]) s.found = s.key[tid * PER + j];
      at += v[j];
    }
    __syncthreads();
    last = s.found;
    if (last == 0) {                 // not where the bins said: never expected
      sample_any<X>(row, a, t, s.request, wt, s);
      return;
    }
    // the listed ones that stay, to their chunks
    for (int i = tid; i < n; i += TPB) {
      const u64 key = s.key[i];
      const float x = key_value(key);
      if (key < last || x < t_mp) continue;
      const int col = int(key_index(key));
      atomicAdd(&s.fast.chunk[col < first ? 0 : col >= tail_col ? chunks - 1 : 1 + (col - first) / CHUNK], wt.whole(x));
    }
    __syncthreads();
  }
  if (cut && mode == TIED) {
    // a crowd of one value, of which the first `need` stay, in the order of the index
    constexpr int PER = CHUNKS / TPB;
    const float x = value_of(low_order);
    const u64 each = wt.whole(x), target = by_count ? u64(s.request.k) : start_of(s.request.p, sum_of_all);
    u64 certain = 0, mine = 0, ties;
    for (int i = tid; i < chunks; i += TPB) certain += s.fast.chunk[i];
    scan_before(certain, s, certain);
    if (by_count) certain = s.count_before;
    for (int j = 0; j < PER; ++j) mine += tid * PER + j < chunks ? s.fast.bin[tid * PER + j] : 0;
    u64 at = scan_before(mine, s, ties);
    const u64 need = target <= certain ? 0 : by_count ? target - certain : each ? (target - certain + each - 1) / each : 0;
    if (need == 0 || need > ties) {  // never expected
      __syncthreads();
      sample_any<X>(row, a, t, s.request, wt, s);
      return;
    }
    for (int j = 0; j < PER && tid * PER + j < chunks; ++j) {
      const int i = tid * PER + j;
      const u64 n = s.fast.bin[i], stay = at >= need ? 0 : min(n, need - at);
      if (x >= t_mp) s.fast.chunk[i] += stay * each;
      if (at < need && need <= at + n) {
        s.first_bin = i;
        s.before = at;
      }
      at += n;
    }
    __syncthreads();
    int from, to;
    bounds(s.first_bin, from, to);
    bool tie[SHARE];
    mine = 0;
#pragma unroll
    for (int j = 0; j < SHARE; ++j) {
      const int i = from + tid * SHARE + j;
      tie[j] = i < to && order_of(to_f(row[i])) == low_order;
      mine += tie[j];
    }
    at = s.before + scan_before(mine, s, ties);
#pragma unroll
    for (int j = 0; j < SHARE; ++j)
      if (tie[j] && ++at == need) s.found = make_key(x, uint32_t(from + tid * SHARE + j));
    __syncthreads();
    last = s.found;
  }
  // the chunk, and the token in it
  constexpr int PER = CHUNKS / TPB;
  u64 mine = 0, all;
  for (int j = 0; j < PER; ++j) {
    const int i = tid * PER + j;
    mine += i < chunks ? s.fast.chunk[i] : 0;
  }
  u64 at = scan_before(mine, s, all);
  const u64 limit = limit_of(s.request.u, all);
  for (int j = 0; j < PER; ++j) {
    const int i = tid * PER + j;
    const u64 v = i < chunks ? s.fast.chunk[i] : 0;
    if (at <= limit && limit < at + v) {
      s.first_bin = i;
      s.before = at;
    }
    at += v;
  }
  __syncthreads();
  int from, to;
  bounds(s.first_bin, from, to);
  u64 v[SHARE], before = s.before;
  mine = 0;
#pragma unroll
  for (int j = 0; j < SHARE; ++j) {
    const int i = from + tid * SHARE + j;
    v[j] = 0;
    if (i < to) {
      const float x = to_f(row[i]);
      if (make_key(x, uint32_t(i)) >= last && x >= t_mp) v[j] = wt.whole(x);
    }
    mine += v[j];
  }
  u64 in_chunk;
  before += scan_before(mine, s, in_chunk);
#pragma unroll
  for (int j = 0; j < SHARE; ++j) {
    const int i = from + tid * SHARE + j;
    if (before <= limit && limit < before + v[j]) put_drawn(a, t, i, to_f(row[i]), wt, v[j], all, wt.log_factor());
    before += v[j];
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
  // a row's results are written while other rows are read; in the very place of its random number or of a setting they are not in the way
  const int token_size = type_size(id_type);
  const void *results[] = {token, logprob}, *inputs[] = {u, scale, top_k, top_p, min_p};
  for (int i = 0; i < 2; ++i) {
    const int size = i ? 4 : token_size;
    if (share_vector(results[i], T, size, logits, T, V, ld, type_size(type))) return MV_ERR_INVALID_ARG;
    for (const void* p : inputs)
      if (share_vector(results[i], T, size, p, 1, T, T, 4) && !(p == results[i] && size == 4)) return MV_ERR_INVALID_ARG;
  }
  if (share_vector(token, T, token_size, logprob, 1, T, T, 4)) return MV_ERR_INVALID_ARG;
  SampleArgs a;
  a.V = V; a.ld = ld; a.u = u; a.scale = scale; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.token = token; a.id_type = id_type; a.logprob = logprob;
  a.unit = 0x1p51;                   // one of 2^52 has to fit the lower bits of a double
  for (int64_t n = 1024; n < V; n *= 2) a.unit *= 0.5;
  return with_type(type, [&](auto x) {
    using X = decltype(x);
    const int64_t vecs = V / Vec<X>::N;
    a.chunks = V / CHUNK + 10 <= CHUNKS;
    // As many CTAs per row as fill the device twice (requests of different kinds end at different times), a step or more for each: 256 rows of
    // 131072 bf16, mixed requests: 94 us, once 102, four times 119; all of one kind, top k 50 and top p 0.9, 38, 29 and 60, top p alone
    // 156, 157 and 224.  Rows of 256 KB and more are shared by two at least, as mixed requests end unevenly (1024 rows: 230 us, by one
    // CTA each 271; 600 with nothing cut 129 and 140; of 200 KB, 1024 of f32 112 and 102, 600 of bf16 108 and 115).
    const int least = vecs >= 16 * TPB * U ? 2 : 1;
    int ctas = MOST_CTAS;
    while (ctas > least && (T * ctas > 2 * 148 * RESIDENT || vecs < int64_t(ctas) * TPB * U)) ctas /= 2;
    if (T * ctas >= lim) return int(MV_ERR_INVALID_ARG);
    const int64_t n_steps = ((vecs + ctas - 1) / ctas + CHUNK / Vec<X>::N + TPB * U - 1) / (TPB * U);
    a.steps = int((n_steps + GROUPS - 1) / GROUPS);
    if (a.steps < 1) a.steps = 1;
    auto* kernel = k_sample<X>;
    static SmemLimit limit;
    if (!allow_smem(kernel, int(sizeof(Smem)), &limit)) return int(MV_ERR_CUDA);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(T * ctas));
    cfg.blockDim = dim3(TPB);
    cfg.dynamicSmemBytes = sizeof(Smem);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = unsigned(ctas);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = ctas > 1;
    const bool ok = cudaLaunchKernelEx(&cfg, kernel, static_cast<const X*>(logits), a) == cudaSuccess;
    return cuda_ok() == MV_OK && ok ? int(MV_OK) : int(MV_ERR_CUDA);
  });
}

}  // extern "C"
