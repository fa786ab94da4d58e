// mv_norm.cu -- layer norm of rows, for sm_100a.
//
// Forward: mu = mean x, then v = mean (x - mu)^2 of the same registers (one reading of memory; no difference of large sums; what mu is
// off is put right by the same pass), r = 1 / sqrt(v + eps), y = (x - mu) r w + b.  Backward, with n = (x - mu) r and h = dy w: the two sums of h and h n in one reduction, dx = r (h -
// mean h - n mean(h n)); the sums over rows of dy n and dy stay in the registers of the thread that owns the columns, CTA by CTA, and
// a second kernel adds the CTAs' sums up in their order.  Memory bounds both where rows are many and lie on 16-byte boundaries: 65536 x
// 2048 bf16 94 us (5.7 TB/s in and out), its gradient 155 us (5.2 TB/s, 6 us of it the second kernel); 32768 x 4096 99 and 163, 32768 x 2048
// f32 90 and 148.  A few thousand short rows are bound by latency: 2048 x 512 6 (8 from call to call) and 12.6 us.  Times are those of calls that follow one another for
// half a second, at the power limit; in short runs memory-bound ones take up to a tenth less (90 and 141 us), and where a comment compares two
// forms, both were timed like that.
//
// Edges: forward, rows of more than 25600 columns (parameters do not fit shared memory), of f32 more than 16384, off the boundaries from 16384
// on, take k_norm_long, three readings: 4096 x 28000 bf16 236 us (floor 70), 4096 x 16384 f32 off the boundaries 162 (16381 columns: 133,
// floor 82).  Gradient: see k_norm_grad.

#include "mv_norm.cuh"

namespace {

struct NormArgs {
  int64_t T, D, ldx, ldy;
  const void *weight, *bias;
  int w_type;
  float eps;
  float *mean, *rstd;
  int64_t per;                       // rows per CTA
};

// Threads at work at once decide how many bytes are on their way: CTAs per multiprocessor that the registers allow.
constexpr int norm_resident(int elements, bool wide) { return elements > 16 ? (wide ? 1 : 2) : wide ? 2 : elements > 8 ? 4 : 6; }

// Rows on 16-byte boundaries.  The next row's vectors are on their way while a row is worked on, parameters wait in shared memory in 32
// bits (they may lie anywhere in memory).  Eight vectors a lane where there are many rows: 16 shuffles a row instead of 80 for one.
template <typename X, int L, int NV>
__global__ void __launch_bounds__(L > 32 ? WIDE_TPB : NORM_TPB, norm_resident(NV * Unit<X, true>::N, L > 32)) k_norm(const X* x, X* y, const __grid_constant__ NormArgs a) {
  using Un = Unit<X, true>;
  constexpr int N = Un::N, GROUPS = (L > 32 ? WIDE_TPB : NORM_TPB) / L, WARPS = L / 32;
  extern __shared__ float4 params[];         // weights, then biases
  __shared__ float part[3][WIDE_TPB / 32];
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
  auto sum = [&](float v) {
    v = lanes_sum<(L < 32 ? L : 32)>(v);
    if constexpr (WARPS > 1) {
      if ((threadIdx.x & 31) == 0) part[0][threadIdx.x >> 5] = v;
      group_sync<L>(mine);
      v = 0.0f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) v += part[0][mine * WARPS + i];
    }
    return v;
  };
  auto sum_both = [&](float& v, float& w) {
    v = lanes_sum<(L < 32 ? L : 32)>(v);
    w = lanes_sum<(L < 32 ? L : 32)>(w);
    if constexpr (WARPS > 1) {
      if ((threadIdx.x & 31) == 0) {
        part[1][threadIdx.x >> 5] = v;
        part[2][threadIdx.x >> 5] = w;
      }
      group_sync<L>(mine);
      v = w = 0.0f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        v += part[1][mine * WARPS + i];
        w += part[2][mine * WARPS + i];
      }
    }
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
    const float m = sum(add_up(s)) * share;
    const f2 minus = both(-m);
    f2 off = both(0.0f);
    s = off;
    each_pair<X, true, NV>(n, [&](int i, int j, int, bool second) {
      const f2 d = add2(pair_of<X, true>(get, i, j, second), minus);
      off = add2(off, d);
      s = fma2(d, d, s);
    });
    float sum_d = add_up(off), sum_d2 = add_up(s);
    sum_both(sum_d, sum_d2);
    const Centre c = centre(m, sum_d, sum_d2, share, a.eps);
    if (t >= t1) continue;
    const f2 rs2 = both(c.rstd), shift2 = both(c.shift);
    put_pairs<X, true, NV, L>(n, y + t * a.ldy + at * N, [&](int i, int j, int k, bool second) {
      return fma2(fma2(add2(pair_of<X, true>(get, i, j, second), minus), rs2, shift2), param_pair<N, L>(pw, at, units, k, second), param_pair<N, L>(pb, at, units, k, second));
    });
    if (at == 0) {
      if (a.mean) a.mean[t] = c.mean;
      if (a.rstd) a.rstd[t] = c.rstd;
    }
  }
}

// Rows that do not lie on 16-byte boundaries.  The vectors are those of y's row, from its first boundary on (in every row another column); what is
// before and behind them, up to 31 elements, goes to a lane each.  APART: x lies otherwise within 16 bytes, and comes from between
// two of its vectors.  Weight and bias of a column side by side, those of every N-th column together, so that neighbouring lanes
// read neighbouring pairs wherever the vectors begin.  30000 x 1001 bf16: 39 us (element by element 45 to 80, floor 18); bound by instructions, 25 an
// element, half of them for the parameters and the shift.
template <typename X, bool APART, int L, int NV>
__global__ void __launch_bounds__(L > 32 ? WIDE_TPB : NORM_TPB, L > 32 ? 1 : 2) k_norm_any(const X* x, X* y, const __grid_constant__ NormArgs a) {
  constexpr int N = Vec<X>::N, GROUPS = (L > 32 ? WIDE_TPB : NORM_TPB) / L, WARPS = L / 32, SIZE = sizeof(X), ENDS = L < 32 ? 32 / L : 1;
  extern __shared__ float2 pairs[];
  __shared__ float part[3][WIDE_TPB / 32];
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
        // in place (never APART) the rows are written by this kernel, which the non-coherent path does not allow for
        if constexpr (APART) {
          next[i] = __ldg(p + i * L);
          more[i] = __ldg(p + i * L + 1);
        } else {
          next[i] = __ldcs(p + i * L);
        }
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
  auto sum = [&](float v) {
    v = lanes_sum<(L < 32 ? L : 32)>(v);
    if constexpr (WARPS > 1) {
      if ((threadIdx.x & 31) == 0) part[0][threadIdx.x >> 5] = v;
      group_sync<L>(mine);
      v = 0.0f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) v += part[0][mine * WARPS + i];
    }
    return v;
  };
  auto sum_both = [&](float& v, float& w) {
    v = lanes_sum<(L < 32 ? L : 32)>(v);
    w = lanes_sum<(L < 32 ? L : 32)>(w);
    if constexpr (WARPS > 1) {
      if ((threadIdx.x & 31) == 0) {
        part[1][threadIdx.x >> 5] = v;
        part[2][threadIdx.x >> 5] = w;
      }
      group_sync<L>(mine);
      v = w = 0.0f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        v += part[1][mine * WARPS + i];
        w += part[2][mine * WARPS + i];
      }
    }
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
    const float m = sum(add_up(s)) * share;
    const f2 minus = both(-m);
    f2 off = both(0.0f);
    s = off;
#pragma unroll
    for (int i = 0; i < ENDS; ++i) {
      const f2 d = pack2(at + i * L < ends ? end[i] - m : 0.0f, 0.0f);
      off = add2(off, d);
      s = fma2(d, d, s);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i < n)
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
          const f2 d = add2(Vec<X>::pair(u[i], j), minus);
          off = add2(off, d);
          s = fma2(d, d, s);
        }
    float sum_d = add_up(off), sum_d2 = add_up(s);
    sum_both(sum_d, sum_d2);
    const Centre c = centre(m, sum_d, sum_d2, share, a.eps);
    if (t >= t1) continue;
    const f2 rs2 = both(c.rstd), shift2 = both(c.shift);
    auto place = [&](int column) { return column % N * columns + column / N; };
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
        unpack2(fma2(fma2(add2(Vec<X>::pair(u[i], j), minus), rs2, shift2), pack2(p.x, q.x), pack2(p.y, q.y)), o[2 * j], o[2 * j + 1]);
      }
      __stcs(reinterpret_cast<uint4*>(now.y + now.first) + v, pack_vec<X>(o));
    }
#pragma unroll
    for (int i = 0; i < ENDS; ++i) {
      const int e = at + i * L;
      if (e >= ends) break;
      const int column = e < now.first ? e : now.nv * N + e;
      const float2 p = pairs[place(column)];
      now.y[column] = from_f<X>(fmaf(fmaf(end[i] - m, c.rstd, c.shift), p.x, p.y));
    }
    if (at == 0) {
      if (a.mean) a.mean[t] = c.mean;
      if (a.rstd) a.rstd[t] = c.rstd;
    }
  }
}

template <typename X>
__global__ void __launch_bounds__(LONG_TPB) k_norm_long(const X* x, X* y, const __grid_constant__ NormArgs a) {
  __shared__ float sh[LONG_TPB / 32];
  const int64_t t = blockIdx.x;
  const X* row = x + t * a.ldx;
  X* out = y + t * a.ldy;
  float s = 0.0f;
  for (int64_t i = threadIdx.x; i < a.D; i += LONG_TPB) s += to_f(row[i]);
  const float share = 1.0f / float(a.D), m = cta_sum(s, sh) * share;
  float off = 0.0f;
  s = 0.0f;
  for (int64_t i = threadIdx.x; i < a.D; i += LONG_TPB) {
    const float d = to_f(row[i]) - m;
    off += d;
    s = fmaf(d, d, s);
  }
  off = cta_sum(off, sh);
  const Centre c = centre(m, off, cta_sum(s, sh), share, a.eps);
  for (int64_t i = threadIdx.x; i < a.D; i += LONG_TPB)
    out[i] = from_f<X>(fmaf(fmaf(to_f(row[i]) - m, c.rstd, c.shift), parameter(a.weight, a.w_type, i, 1.0f), parameter(a.bias, a.w_type, i, 0.0f)));
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[t] = c.mean;
    if (a.rstd) a.rstd[t] = c.rstd;
  }
}

constexpr int WAVES = 3;

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
  // the statistics of a row are written while others are read and written
  for (const float* p : {mean, rstd})
    if (share_vector(p, T, 4, x, T, D, ldx, size) || share_vector(p, T, 4, y, T, D, ldy, size) || share_vector(p, T, 4, weight, 1, D, D, wsize) ||
        share_vector(p, T, 4, bias, 1, D, D, wsize))
      return MV_ERR_INVALID_ARG;
  if (share_vector(mean, T, 4, rstd, 1, T, T, 4)) return MV_ERR_INVALID_ARG;
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
      if (smem > SMEM_UNASKED && !allow_smem(kernel, int(smem), limit)) return int(MV_ERR_CUDA);
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

}  // extern "C"
