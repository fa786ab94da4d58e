// mv_norm_grad.cu -- the gradients of layer norm, for sm_100a; what bounds them is said in mv_norm.cu.

#include "mv_norm.cuh"

namespace {

struct NormGradArgs {
  int64_t T, D, lddy, ldx, lddx;
  const void* weight;
  int w_type;
  const float *mean, *rstd;
  float *dweight, *dbias, *part;      // part: [CTAs][2][D]
  int accumulate, parts;
  int64_t per;                       // rows per CTA
  int stages, image;
};

// 16 bytes to shared memory, or as many zeros.
__device__ __forceinline__ void fetch(void* to, const void* from, bool any) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(uint32_t(__cvta_generic_to_shared(to))), "l"(from), "r"(any ? 16 : 0) : "memory");
}
__device__ __forceinline__ void fetches_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void fetched(int behind) {        // all but the last `behind` groups of copies have come
  if (behind == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (behind == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// A row that lies anywhere, as the vectors in which its bytes are: L lanes copy them, and it begins (address mod 16) bytes into `to`.  The
// neighbouring rows' bytes may come with it; what is outside the T rows [lo, hi) does not.
inline int image_bytes(int64_t D, int size) { return int((D * size + 15) / 16 + 1) * 16; }
template <typename X, int L> __device__ __forceinline__ void fetch_row(char* to, const X* row, int D, int at, const X* lo, const X* hi) {
  const char* a = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(row) & ~uintptr_t(15));
  const int vecs = int((reinterpret_cast<const char*>(row + D) - a + 15) / 16);
  if (a >= reinterpret_cast<const char*>(lo) && a + 16 * vecs <= reinterpret_cast<const char*>(hi)) {
#pragma unroll 2
    for (int i = at; i < vecs; i += L) fetch(to + 16 * i, a + 16 * i, true);
  } else {                           // the first and the last row
    for (int i = at; i < D; i += L) const_cast<X*>(reinterpret_cast<const X*>(to + (reinterpret_cast<uintptr_t>(row) & 15)))[i] = row[i];
  }
}
template <typename X> __device__ __forceinline__ const X* in_image(const char* image, const X* row) {
  return reinterpret_cast<const X*>(image + (reinterpret_cast<uintptr_t>(row) & 15));
}

// R rows at a time; a thread owns its columns' sums over rows.  The units of x and dy travel through a thread's own places in
// shared memory, a.stages deep, so that nothing waits for them but the thread itself; of rows that lie anywhere, as images that their lanes
// share.  One barrier for R rows.  8191 x 1001 f32 with pitches of 1003 and 1001: 27 us for 98 MB, half of it start, end and the second
// kernel; 30000 x 1001 bf16 55 us, bound by instructions (an element at a time is read, weighed twice and written).
// Edges: f32 from 8200 columns on has room for one stage, so that a row's loads are not covered by another's work (8192 x 8192 140 us, 8200 columns
// 181, floor 123); f32 off the boundaries has no room for two images from 11517 columns on and takes k_norm_grad_long, as everything
// above 16384 columns does: single elements, sums over rows in memory (4096 x 11500 f32 121 us, 11520 columns 476, floor 86; 4096 x
// 20480 bf16 998, floor 77).
template <int L> constexpr int GRAD_THREADS = L > NORM_TPB ? L : NORM_TPB;

template <typename X, bool VEC, int L, int NV, int R>
__global__ void __launch_bounds__(GRAD_THREADS<L>, L > NORM_TPB ? 1 : 2) k_norm_grad(const X* dy, const X* x, X* dx, const __grid_constant__ NormGradArgs a) {
  using Un = Unit<X, VEC>;
  constexpr int N = Un::N, PAIRS = NV * N / 2, THREADS = GRAD_THREADS<L>, GROUPS = THREADS / L, WARPS = L / 32, STAGE = R * NV * 2 * THREADS;
  extern __shared__ float4 shared[];         // the ring (or the images), weights, laid out as above; at the end the groups' sums
  __shared__ float part[2][2 * R][THREADS / 32];
  const int D = int(a.D), units = D / N, tid = threadIdx.x, mine = tid / L, at = tid % L;
  const int n = units > at ? (units - at - 1) / L + 1 : 0;
  Un* ring = reinterpret_cast<Un*>(shared);
  char* images = reinterpret_cast<char*>(shared) + mine * (R * 2) * a.image;       // of a group; GROUPS of them for each stage
  const int stage = VEC ? STAGE * 16 : GROUPS * R * 2 * a.image;
  float* pw = reinterpret_cast<float*>(reinterpret_cast<char*>(shared) + a.stages * stage);
  const int64_t t0 = blockIdx.x * a.per, t1 = min(a.T, t0 + a.per);
  constexpr int STEP = GROUPS * R;
  auto row = [&](int64_t r0, int r) { return r0 + r * GROUPS + mine; };
  auto issue = [&](int64_t r0, int slot) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t t = row(r0, r);
      if constexpr (VEC) {
        const int any = t < t1 ? n : 0;
        const X *px = x + t * a.ldx + at * N, *py = dy + t * a.lddy + at * N;
        Un* to = ring + slot * STAGE + r * NV * 2 * THREADS + tid;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          fetch(to + i * 2 * THREADS, i < any ? px + i * L * N : x, i < any);
          fetch(to + (i * 2 + 1) * THREADS, i < any ? py + i * L * N : dy, i < any);
        }
      } else if (t < t1) {
        char* to = images + slot * stage + r * 2 * a.image;
        fetch_row<X, L>(to, x + t * a.ldx, D, at, x, x + (a.T - 1) * a.ldx + D);
        fetch_row<X, L>(to + a.image, dy + t * a.lddy, D, at, dy, dy + (a.T - 1) * a.lddy + D);
      }
    }
    fetches_end();
  };
  float mu[R], rs[R];
  auto statistics = [&](int64_t r0) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t t = row(r0, r);
      mu[r] = t < t1 ? a.mean[t] : 0.0f;
      rs[r] = t < t1 ? a.rstd[t] : 0.0f;
    }
  };
  for (int s = 0; s + 1 < a.stages; ++s) issue(t0 + s * STEP, s);
  statistics(t0);
  put_params<N>(pw, a.weight, a.w_type, 1.0f, D, units);
  f2 dw[PAIRS], db[PAIRS];
#pragma unroll
  for (int k = 0; k < PAIRS; ++k) dw[k] = db[k] = both(0.0f);
  __syncthreads();
  const float share = 1.0f / float(D);
  int flip = 0, slot = 0;
  for (int64_t r0 = t0; r0 < t1; r0 += STEP) {
    if constexpr (VEC) {
      issue(r0 + (a.stages - 1) * STEP, slot == 0 ? a.stages - 1 : slot - 1);
      fetched(a.stages - 1);
    } else {
      fetched(a.stages - 2);
      group_sync<L>(mine);           // the rows have come, and the ones before have been read
      issue(r0 + (a.stages - 1) * STEP, slot == 0 ? a.stages - 1 : slot - 1);
    }
    // x (0) or dy (1) of row r
    auto of = [&](int r, int which) {
      if constexpr (VEC) {
        const Un* from = ring + slot * STAGE + (r * NV * 2 + which) * THREADS + tid;
        return [from](int i) -> const Un& { return from[i * 2 * THREADS]; };
      } else {
        const int64_t t = row(r0, r);
        const X* from = in_image(images + slot * stage + (r * 2 + which) * a.image, which ? dy + t * a.lddy : x + t * a.ldx) + at;
        return [from](int i) { return Un{from[i * L]}; };
      }
    };
    float s[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      f2 s0 = both(0.0f), s1 = s0;
      const int some = VEC || row(r0, r) < t1 ? n : 0;
      const f2 minus = both(-mu[r]), rs2 = both(rs[r]);
      auto gx = of(r, 0), gy = of(r, 1);
      each_pair<X, VEC, NV>(some, [&](int i, int j, int k, bool second) {
        const f2 vx = pair_of<X, VEC>(gx, i, j, second), vy = pair_of<X, VEC>(gy, i, j, second);
        const f2 nn = mul2(add2(vx, minus), rs2), h = mul2(vy, param_pair<N, L>(pw, at, units, k, second));
        s0 = add2(s0, h);
        s1 = fma2(h, nn, s1);
        dw[k] = fma2(vy, nn, dw[k]);
        db[k] = add2(db[k], vy);
      });
      s[2 * r] = add_up(s0);
      s[2 * r + 1] = add_up(s1);
    }
    if (dx) {
#pragma unroll
      for (int j = 0; j < 2 * R; ++j) s[j] = lanes_sum<(L < 32 ? L : 32)>(s[j]);
      if constexpr (WARPS > 1) {
        if ((tid & 31) == 0)
#pragma unroll
          for (int j = 0; j < 2 * R; ++j) part[flip][j][tid >> 5] = s[j];
        group_sync<L>(mine);
#pragma unroll
        for (int j = 0; j < 2 * R; ++j) {
          s[j] = 0.0f;
#pragma unroll
          for (int i = 0; i < WARPS; ++i) s[j] += part[flip][j][mine * WARPS + i];
        }
        flip ^= 1;
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int64_t t = row(r0, r);
        if (t >= t1) continue;
        const f2 minus = both(-mu[r]), rs2 = both(rs[r]), m0 = both(-s[2 * r] * share), m1 = both(-s[2 * r + 1] * share);
        auto gx = of(r, 0), gy = of(r, 1);
        put_pairs<X, VEC, NV, L>(n, dx + t * a.lddx + at * N, [&](int i, int j, int k, bool second) {
          const f2 nn = mul2(add2(pair_of<X, VEC>(gx, i, j, second), minus), rs2);
          return mul2(fma2(nn, m1, fma2(pair_of<X, VEC>(gy, i, j, second), param_pair<N, L>(pw, at, units, k, second), m0)), rs2);
        });
      }
    }
    statistics(r0 + STEP);
    slot = slot + 1 == a.stages ? 0 : slot + 1;
  }
  if (!a.part) return;
  float* out = a.part + int64_t(blockIdx.x) * 2 * D;
  float* sums = GROUPS == 1 ? out : reinterpret_cast<float*>(shared) + mine * 2 * D;
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PAIRS; ++k) {
    float w[2], b[2];
    unpack2(dw[k], w[0], w[1]);
    unpack2(db[k], b[0], b[1]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int c = N == 1 ? at + (2 * k + e) * L : (at + k / (N / 2) * L) * N + k % (N / 2) * 2 + e;
      if (c < D) {
        sums[c] = w[e];
        sums[D + c] = b[e];
      }
    }
  }
  if (GROUPS == 1) return;
  __syncthreads();
  for (int c = tid; c < 2 * D; c += THREADS) {
    float v = 0.0f;
    for (int g = 0; g < GROUPS; ++g) v += reinterpret_cast<const float*>(shared)[g * 2 * D + c];
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

// The CTAs' sums, 32 columns (of 2 D) per CTA, each by 32 threads in turn.
constexpr int JOIN = 32;
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

constexpr int64_t MOST_PARTS = 148 * 2;
inline int64_t norm_parts(int64_t T, int64_t D) {
  int64_t n = (int64_t(1) << 25) / D;
  if (n > MOST_PARTS) n = MOST_PARTS;
  if (n > T) n = T;
  return n < 1 ? 1 : n;
}

}  // namespace

extern "C" {

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
  for (const float* p : {mean, rstd})
    if (share_vector(p, T, 4, dx, T, D, lddx, size)) return MV_ERR_INVALID_ARG;
  if (dweight || dbias) {
    const size_t need = mv_layer_norm_grad_workspace_bytes(T, D);
    if (!workspace || workspace_bytes < need) return MV_ERR_WORKSPACE;
    const int64_t words = int64_t(need / 4);
    if (share_vector(workspace, words, 4, x, T, D, ldx, size) || share_vector(workspace, words, 4, dy, T, D, lddy, size) ||
        share_vector(workspace, words, 4, dx, T, D, lddx, size) || share_vector(workspace, words, 4, weight, 1, D, D, wsize))
      return MV_ERR_INVALID_ARG;
    for (const float* p : {mean, rstd})
      if (share_vector(p, T, 4, workspace, 1, words, words, 4)) return MV_ERR_INVALID_ARG;
    for (const float* p : {dweight, dbias})
      if (share_vector(p, D, 4, workspace, 1, words, words, 4)) return MV_ERR_INVALID_ARG;
  }
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
      // (images of rows of 32 elements a lane leave room for one CTA only where they are of 4 bytes)
      constexpr int N = Unit<X, VEC>::N, LEAST = VEC ? 1 : 4, LIKED = (VEC || sizeof(X) == 4 ? 16 : 32) / N, MOST = 32 / N;
      Shape s;
      if (!norm_shape(D / N, T, 8, 512, LEAST, LIKED, MOST, &s)) return -1;
      return with_shape<8, 512, LEAST, LIKED, MOST, 8>(s, [&](auto lanes, auto nv) {
        constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value, THREADS = GRAD_THREADS<L>, GROUPS = THREADS / L;
        constexpr int R = NV * N > 16 ? 1 : VEC ? (NV < 4 ? 4 / NV : 1) : (NV < 16 ? 2 : 1);
        a.image = VEC ? 0 : image_bytes(D, size);
        const int64_t stage = VEC ? int64_t(R) * NV * 2 * THREADS * 16 : int64_t(GROUPS) * R * 2 * a.image;
        // Two CTAs of 256 threads with two stages each come before three stages, and more than a few rows for each before more CTAs, whose
        // sums are written and read again.
        int64_t parts = L > NORM_TPB ? 1 : 2;
        const int64_t least_smem = 2 * stage + 4 * D > GROUPS * 8 * D ? 2 * stage + 4 * D : GROUPS * 8 * D;
        if (parts * (least_smem + 2048) > 227 * 1024) parts = 1;
        for (a.stages = 3; a.stages && parts * (a.stages * stage + 4 * D + 2048) > 227 * 1024; --a.stages) {}
        if (a.stages < (VEC ? 1 : 2)) return -1;
        parts *= 148;
        const int64_t few = T * size / 16 > 64 ? T * size / 16 : 64;
        if (parts > few) parts = few;
        if (parts > most_parts) parts = most_parts;
        a.per = ((T + parts - 1) / parts + GROUPS - 1) / GROUPS * GROUPS;
        a.parts = int((T + a.per - 1) / a.per);
        const int64_t turns = (a.per + GROUPS * R - 1) / (GROUPS * R);
        if (a.stages > turns) a.stages = turns > 1 || VEC ? int(turns) : 2;
        size_t smem = size_t(a.stages * stage + 4 * D);
        if (GROUPS > 1 && smem < size_t(GROUPS * 8 * D)) smem = size_t(GROUPS * 8 * D);
        auto* kernel = k_norm_grad<X, VEC, L, NV, R>;
        static SmemLimit limit;
        if (smem > SMEM_UNASKED && !allow_smem(kernel, int(smem), &limit)) return int(MV_ERR_CUDA);
        kernel<<<unsigned(a.parts), THREADS, smem, st>>>(yp, xp, dxp, a);
        return cuda_ok();
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
