// mv_clip.cu -- norms over many tensors, one per group, and clipping in place or into the workers' rows, for sm_100a.
#include "mv_lm.cuh"

#include <math.h>
#include <stdlib.h>

namespace {

constexpr int TPB = 256;
constexpr int CHUNK = 8192;          // elements per chunk

struct Chunk {
  void* ptr;                         // first element
  int64_t dst;                       // its place in the group's row
  int32_t n;
  int32_t type;
  int32_t group;
  int32_t pad;
};

struct Layout { size_t chunks, partial, first, coef, total; int64_t n; };

inline bool clip_layout(const int64_t* numel, int n_tensors, int n_groups, Layout* L) {
  if (n_tensors < 0 || (n_tensors > 0 && !numel) || n_groups < 1 || n_groups >= (1 << 20)) return false;
  L->n = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (numel[i] < 0 || numel[i] >= (int64_t(1) << 40)) return false;
    L->n += (numel[i] + CHUNK - 1) / CHUNK;
  }
  if (L->n >= (int64_t(1) << 31)) return false;
  size_t o = 0;
  L->chunks = o;  o = align_up(o + size_t(L->n) * sizeof(Chunk), 256);
  L->first = o;   o = align_up(o + size_t(n_groups + 1) * 4, 256);
  L->partial = o; o = align_up(o + size_t(L->n) * 8, 256);
  L->coef = o;    o = align_up(o + size_t(n_groups) * 4, 256);
  L->total = o;
  return true;
}

__device__ double block_sum(double x, double* sh) {
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
  __syncthreads();
  x = sh[0];
  for (int i = 1; i < TPB / 32; ++i) x += sh[i];
  return x;
}

template <typename X> __device__ double chunk_sum(const X* x, int n) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += TPB) { const double v = to_f(x[i]); s = fma(v, v, s); }
  return s;
}

__global__ void __launch_bounds__(TPB) k_clip_sum(const Chunk* __restrict__ chunks, double* __restrict__ partial) {
  __shared__ double sh[TPB / 32];
  const Chunk c = chunks[blockIdx.x];
  double s = c.type == MV_F32 ? chunk_sum(static_cast<const float*>(c.ptr), c.n)
           : c.type == MV_BF16 ? chunk_sum(static_cast<const __nv_bfloat16*>(c.ptr), c.n)
                               : chunk_sum(static_cast<const __half*>(c.ptr), c.n);
  s = block_sum(s, sh);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ void __launch_bounds__(TPB) k_clip_norm(const double* __restrict__ partial, const int32_t* __restrict__ first, float max_norm,
                                                    float* __restrict__ norms, float* __restrict__ coef) {
  __shared__ double sh[TPB / 32];
  const int g = blockIdx.x;
  double s = 0.0;
  for (int i = first[g] + threadIdx.x; i < first[g + 1]; i += TPB) s += partial[i];
  s = block_sum(s, sh);
  if (threadIdx.x == 0) {
    const double n = sqrt(s);
    if (norms) norms[g] = float(n);
    coef[g] = n > double(max_norm) && !isinf(n) ? float(double(max_norm) / n) : 1.0f;
  }
}

template <typename X> __device__ void chunk_scale(X* x, int n, float c) {
  for (int i = threadIdx.x; i < n; i += TPB) x[i] = from_f<X>(to_f(x[i]) * c);
}
template <typename X> __device__ void chunk_pack(const X* x, int n, float c, float* dst) {
  for (int i = threadIdx.x; i < n; i += TPB) dst[i] = to_f(x[i]) * c;
}

__global__ void __launch_bounds__(TPB) k_clip_apply(const Chunk* __restrict__ chunks, const float* __restrict__ coef, float* rows, int64_t ld) {
  const Chunk c = chunks[blockIdx.x];
  const float f = coef[c.group];
  if (rows) {
    float* dst = rows + c.group * ld + c.dst;
    if (c.type == MV_F32) chunk_pack(static_cast<const float*>(c.ptr), c.n, f, dst);
    else if (c.type == MV_BF16) chunk_pack(static_cast<const __nv_bfloat16*>(c.ptr), c.n, f, dst);
    else chunk_pack(static_cast<const __half*>(c.ptr), c.n, f, dst);
  } else if (f != 1.0f) {
    if (c.type == MV_F32) chunk_scale(static_cast<float*>(c.ptr), c.n, f);
    else if (c.type == MV_BF16) chunk_scale(static_cast<__nv_bfloat16*>(c.ptr), c.n, f);
    else chunk_scale(static_cast<__half*>(c.ptr), c.n, f);
  }
}

}  // namespace

struct mv_clip {
  int64_t n;                         // chunks
  int n_groups;
  int64_t longest;                   // elements of the longest group
  uintptr_t lo, hi;                  // addresses that the tensors span
  int n_tensors;
  struct Span { uintptr_t lo, hi; }* spans;      // host: the bytes of each tensor
  Chunk* chunks;
  int32_t* first;
  double* partial;
  float* coef;
};

namespace {

// Whether the rows and one of the tensors share bytes.
bool overlaps(const mv_clip* p, const float* rows, int64_t ld) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(rows), hi = lo + (size_t(p->n_groups - 1) * ld + p->longest) * 4;
  if (hi <= p->lo || lo >= p->hi) return false;
  for (int i = 0; i < p->n_tensors; ++i)
    if (p->spans[i].lo < hi && lo < p->spans[i].hi) return true;
  return false;
}

int clip_norms(mv_clip* p, cudaStream_t st, float max_norm, float* norms) {
  if (p->n > 0) k_clip_sum<<<unsigned(p->n), TPB, 0, st>>>(p->chunks, p->partial);
  k_clip_norm<<<unsigned(p->n_groups), TPB, 0, st>>>(p->partial, p->first, max_norm, norms, p->coef);
  return cuda_ok();
}

}  // namespace

extern "C" {

size_t mv_clip_workspace_bytes(const int64_t* numel, int n_tensors, int n_groups) {
  Layout L;
  return clip_layout(numel, n_tensors, n_groups, &L) ? L.total : 0;
}

int mv_clip_create(mv_clip** out, void* stream, void* const* tensors, const int* types, const int64_t* numel, const int* groups,
                   int n_tensors, int n_groups, void* workspace, size_t workspace_bytes) {
  Layout L;
  if (!out || !clip_layout(numel, n_tensors, n_groups, &L) || (n_tensors > 0 && (!tensors || !types)) || misaligned(workspace, 256))
    return MV_ERR_INVALID_ARG;
  for (int i = 0; i < n_tensors; ++i) {
    const int g = groups ? groups[i] : 0;
    if (!is_value_type(types[i]) || (numel[i] > 0 && !tensors[i]) || misaligned(tensors[i], type_size(types[i])) || g < 0 || g >= n_groups ||
        (i > 0 && groups && g < groups[i - 1]))
      return MV_ERR_INVALID_ARG;
  }
  if (!workspace || workspace_bytes < L.total) return MV_ERR_WORKSPACE;
  mv_clip* p = static_cast<mv_clip*>(calloc(1, sizeof(mv_clip)));
  mv_clip::Span* spans = static_cast<mv_clip::Span*>(calloc(n_tensors ? n_tensors : 1, sizeof(mv_clip::Span)));
  char* host = static_cast<char*>(calloc(1, L.partial));
  if (!p || !spans || !host) { free(p); free(spans); free(host); return MV_ERR_WORKSPACE; }
  char* base = static_cast<char*>(workspace);
  p->n = L.n;
  p->n_groups = n_groups;
  p->n_tensors = n_tensors;
  p->spans = spans;
  p->lo = UINTPTR_MAX;
  p->chunks = reinterpret_cast<Chunk*>(base + L.chunks);
  p->first = reinterpret_cast<int32_t*>(base + L.first);
  p->partial = reinterpret_cast<double*>(base + L.partial);
  p->coef = reinterpret_cast<float*>(base + L.coef);
  Chunk* c = reinterpret_cast<Chunk*>(host + L.chunks);
  int32_t* first = reinterpret_cast<int32_t*>(host + L.first);
  int64_t nc = 0, dst = 0;
  int g = 0;
  first[0] = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const int gi = groups ? groups[i] : 0;
    while (g < gi) { first[++g] = int32_t(nc); dst = 0; }
    for (int64_t o = 0; o < numel[i]; o += CHUNK, ++nc) {
      c[nc].ptr = static_cast<char*>(tensors[i]) + o * type_size(types[i]);
      c[nc].dst = dst + o;
      c[nc].n = int32_t(numel[i] - o < CHUNK ? numel[i] - o : CHUNK);
      c[nc].type = types[i];
      c[nc].group = gi;
    }
    spans[i].lo = reinterpret_cast<uintptr_t>(tensors[i]);
    spans[i].hi = spans[i].lo + size_t(numel[i]) * type_size(types[i]);
    if (numel[i] > 0 && spans[i].lo < p->lo) p->lo = spans[i].lo;
    if (numel[i] > 0 && spans[i].hi > p->hi) p->hi = spans[i].hi;
    dst += numel[i];
    if (dst > p->longest) p->longest = dst;
  }
  while (g < n_groups) first[++g] = int32_t(nc);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool ok = cudaMemcpyAsync(base, host, L.partial, cudaMemcpyHostToDevice, st) == cudaSuccess && cudaStreamSynchronize(st) == cudaSuccess;
  free(host);
  if (!ok) { cudaGetLastError(); mv_clip_destroy(p); return MV_ERR_CUDA; }
  *out = p;
  return MV_OK;
}

int mv_clip_destroy(mv_clip* plan) {
  if (!plan) return MV_ERR_INVALID_ARG;
  free(plan->spans);
  free(plan);
  return MV_OK;
}

int mv_clip_norm(mv_clip* plan, void* stream, float* norms) {
  if (!plan || !norms || misaligned(norms, 4)) return MV_ERR_INVALID_ARG;
  return clip_norms(plan, static_cast<cudaStream_t>(stream), INFINITY, norms);
}

int mv_clip_scale(mv_clip* plan, void* stream, float max_norm, float* norms) {
  if (!plan || !(max_norm >= 0.0f) || misaligned(norms, 4)) return MV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (int rc = clip_norms(plan, st, max_norm, norms)) return rc;
  if (plan->n > 0) k_clip_apply<<<unsigned(plan->n), TPB, 0, st>>>(plan->chunks, plan->coef, nullptr, 0);
  return cuda_ok();
}

int mv_clip_pack(mv_clip* plan, void* stream, float max_norm, float* rows, int64_t ld, float* norms) {
  if (!plan || !(max_norm >= 0.0f) || misaligned(norms, 4) || misaligned(rows, 4) || !rows || ld < plan->longest ||
      overlaps(plan, rows, ld))
    return MV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (int rc = clip_norms(plan, st, max_norm, norms)) return rc;
  if (plan->n > 0) k_clip_apply<<<unsigned(plan->n), TPB, 0, st>>>(plan->chunks, plan->coef, rows, ld);
  return cuda_ok();
}

}  // extern "C"
