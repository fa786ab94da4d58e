// mv_clip.cu -- norms over many tensors, one per group, and clipping in place or into the workers' rows, for sm_100a.
#include "mv_lm.cuh"

#include <math.h>
#include <stdlib.h>

namespace {

// The list is cut into chunks, one CTA each.  A group's factor is known only when all its chunks have been summed, so every
// element is read twice; to read it from memory only once, the list is worked off in stages of whole groups that fit L2: one
// launch scales stage s and sums stage s + 1, mixing the reads of the one with the writes of the other.
constexpr int TPB = 256;
constexpr int CHUNK = 8192;          // elements per chunk: 16 or 32 KB
constexpr int64_t STAGE = int64_t(40) << 20;      // bytes of a stage, or one group

struct Chunk {
  void* ptr;                         // first element
  int64_t dst;                       // its place in the group's row
  int32_t n;
  int32_t type;
  int32_t group;
  int32_t pad;
};

struct Layout { size_t chunks, first, partial, ticket, coef, total; int64_t n; };

inline bool clip_layout(const int64_t* numel, int n_tensors, int n_groups, Layout* L) {
  if (n_tensors < 0 || (n_tensors > 0 && !numel) || n_groups < 1 || n_groups >= (1 << 20)) return false;
  L->n = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (numel[i] < 0 || numel[i] >= (int64_t(1) << 40)) return false;
    L->n += (numel[i] + CHUNK - 1) / CHUNK;
  }
  if (L->n >= (int64_t(1) << 30)) return false;
  size_t o = 0;
  L->chunks = o;  o = align_up(o + size_t(L->n) * sizeof(Chunk), 256);
  L->first = o;   o = align_up(o + size_t(n_groups + 1) * 4, 256);
  L->ticket = o;  o = align_up(o + size_t(n_groups) * 4, 256);      // what the host fills ends here
  L->partial = o; o = align_up(o + size_t(L->n) * 8, 256);
  L->coef = o;    o = align_up(o + size_t(n_groups) * 4, 256);
  L->total = o;
  return true;
}

struct ClipArgs {
  const Chunk* chunks;
  const int32_t* first;              // [groups + 1] first chunk of each group
  uint32_t* ticket;                  // [groups] chunks summed so far; back to 0 with the last one
  double* partial;
  float *coef, *norms;
  float max_norm;
  float* rows;                       // pack: the rows; null: in place
  int64_t ld;
  int n_groups;
  int apply0, n_apply, sum0, n_sum;  // chunks to scale and chunks to sum in this launch
  int empty;                         // the first launch also deals with groups that have no chunk
};

// 16 bytes of a chunk as numbers.
template <typename X> constexpr int PER = 16 / int(sizeof(X));
template <typename X> __device__ __forceinline__ void widen(const uint4& u, float (&f)[PER<X>]) {
  X x[PER<X>];
  memcpy(x, &u, 16);
#pragma unroll
  for (int i = 0; i < PER<X>; ++i) f[i] = to_f(x[i]);
}

// Elements before the first 16-byte boundary.
template <typename X> __device__ __forceinline__ int head_of(const X* x, int n) {
  return min(n, int((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / int(sizeof(X)));
}

// Sum of squares of a chunk, this thread's part.  64 bits: a square of 32 bits has no room below 1e-19 or above 1e19.
template <typename X> __device__ double chunk_sum(const X* x, int n) {
  constexpr int V = CHUNK / PER<X> / TPB;           // vectors per thread, all on their way at once
  const int head = head_of(x, n), nv = (n - head) / PER<X>, tail = head + nv * PER<X>;
  const uint4* p = reinterpret_cast<const uint4*>(x + head);
  uint4 u[V];
#pragma unroll
  for (int i = 0; i < V; ++i) u[i] = i * TPB + int(threadIdx.x) < nv ? __ldg(p + i * TPB + threadIdx.x) : make_uint4(0, 0, 0, 0);
  double s = 0.0;
  if (int(threadIdx.x) < head + n - tail) {
    const double v = to_f(x[int(threadIdx.x) < head ? int(threadIdx.x) : tail + int(threadIdx.x) - head]);
    s = v * v;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float f[PER<X>];
    widen<X>(u[i], f);
#pragma unroll
    for (int j = 0; j < PER<X>; ++j) { const double v = f[j]; s = fma(v, v, s); }
  }
  return s;
}

__device__ double block_sum(double x, double* sh) {
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
  __syncthreads();
  x = sh[0];
  for (int i = 1; i < TPB / 32; ++i) x += sh[i];
  return x;
}

__device__ __forceinline__ void put_norm(const ClipArgs& a, int g, double s) {
  const double n = sqrt(s);
  if (a.norms) a.norms[g] = float(n);
  a.coef[g] = n > double(a.max_norm) && !isinf(n) ? float(double(a.max_norm) / n) : 1.0f;
}

__device__ void sum_chunk(const ClipArgs& a, int i) {
  __shared__ double sh[TPB / 32];
  __shared__ int s_last;
  const Chunk c = a.chunks[i];
  double s = c.type == MV_F32 ? chunk_sum(static_cast<const float*>(c.ptr), c.n)
           : c.type == MV_BF16 ? chunk_sum(static_cast<const __nv_bfloat16*>(c.ptr), c.n)
                               : chunk_sum(static_cast<const __half*>(c.ptr), c.n);
  s = block_sum(s, sh);
  const int c0 = a.first[c.group], c1 = a.first[c.group + 1];
  if (threadIdx.x == 0) {
    __stcg(a.partial + i, s);
    __threadfence();
    s_last = atomicAdd(a.ticket + c.group, 1u) == uint32_t(c1 - c0 - 1);
  }
  __syncthreads();
  if (!s_last) return;
  // the CTA that finishes the group adds its chunks up, always in the same order
  __threadfence();
  s = 0.0;
  for (int k = c0 + threadIdx.x; k < c1; k += TPB) s += __ldcg(a.partial + k);
  s = block_sum(s, sh);
  if (threadIdx.x == 0) {
    put_norm(a, c.group, s);
    a.ticket[c.group] = 0;
  }
}

// Out of place, to 32 bits.  Source and destination lie alike within 16 bytes: groups of four elements; else one by one, which
// still moves whole lines per warp.
template <typename X> __device__ void chunk_pack(const X* x, int n, float c, float* dst) {
  struct alignas(4 * sizeof(X)) Four { X v[4]; };
  const int to16 = int((16 - (reinterpret_cast<uintptr_t>(dst) & 15)) & 15) / 4;
  if ((reinterpret_cast<uintptr_t>(x + to16) & (sizeof(Four) - 1)) == 0) {
    constexpr int V = CHUNK / 4 / TPB;
    const int head = min(n, to16), nv = (n - head) / 4, tail = head + nv * 4;
    const Four* p = reinterpret_cast<const Four*>(x + head);
    float4* q = reinterpret_cast<float4*>(dst + head);
    Four f[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i * TPB + int(threadIdx.x) < nv) f[i] = p[i * TPB + threadIdx.x];
    if (int(threadIdx.x) < head + n - tail) {
      const int e = int(threadIdx.x) < head ? int(threadIdx.x) : tail + int(threadIdx.x) - head;
      dst[e] = to_f(x[e]) * c;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i * TPB + int(threadIdx.x) < nv)
        __stcs(q + i * TPB + threadIdx.x, make_float4(to_f(f[i].v[0]) * c, to_f(f[i].v[1]) * c, to_f(f[i].v[2]) * c, to_f(f[i].v[3]) * c));
  } else {
    constexpr int V = CHUNK / TPB;
    X f[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i * TPB + int(threadIdx.x) < n) f[i] = x[i * TPB + threadIdx.x];
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i * TPB + int(threadIdx.x) < n) __stcs(dst + i * TPB + threadIdx.x, to_f(f[i]) * c);
  }
}

template <typename X> __device__ void chunk_scale(X* x, int n, float c) {
  constexpr int V = CHUNK / PER<X> / TPB;
  const int head = head_of(x, n), nv = (n - head) / PER<X>, tail = head + nv * PER<X>;
  uint4* p = reinterpret_cast<uint4*>(x + head);
  uint4 u[V];
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i * TPB + int(threadIdx.x) < nv) u[i] = p[i * TPB + threadIdx.x];
  if (int(threadIdx.x) < head + n - tail) {
    const int e = int(threadIdx.x) < head ? int(threadIdx.x) : tail + int(threadIdx.x) - head;
    x[e] = from_f<X>(to_f(x[e]) * c);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float f[PER<X>];
    X y[PER<X>];
    widen<X>(u[i], f);
#pragma unroll
    for (int j = 0; j < PER<X>; ++j) y[j] = from_f<X>(f[j] * c);
    memcpy(&u[i], y, 16);
    if (i * TPB + int(threadIdx.x) < nv) __stcs(p + i * TPB + threadIdx.x, u[i]);
  }
}

__device__ void apply_chunk(const ClipArgs& a, int i) {
  const Chunk c = a.chunks[i];
  const float f = __ldcg(a.coef + c.group);
  if (a.rows) {
    float* dst = a.rows + c.group * a.ld + c.dst;
    if (c.type == MV_F32) chunk_pack(static_cast<const float*>(c.ptr), c.n, f, dst);
    else if (c.type == MV_BF16) chunk_pack(static_cast<const __nv_bfloat16*>(c.ptr), c.n, f, dst);
    else chunk_pack(static_cast<const __half*>(c.ptr), c.n, f, dst);
  } else if (f != 1.0f) {
    if (c.type == MV_F32) chunk_scale(static_cast<float*>(c.ptr), c.n, f);
    else if (c.type == MV_BF16) chunk_scale(static_cast<__nv_bfloat16*>(c.ptr), c.n, f);
    else chunk_scale(static_cast<__half*>(c.ptr), c.n, f);
  }
}

__global__ void __launch_bounds__(TPB) k_clip(const __grid_constant__ ClipArgs a) {
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");      // the launch before this one: the factors, and the tensors' other users
  const int n = a.n_apply + a.n_sum;
  if (int(blockIdx.x) >= n) {        // groups without a chunk
    for (int g = threadIdx.x; g < a.n_groups; g += TPB)
      if (a.first[g] == a.first[g + 1]) put_norm(a, g, 0.0);
    return;
  }
  // chunks to scale and chunks to sum, evenly mixed
  const int applied = int(int64_t(blockIdx.x) * a.n_apply / n);
  if (int(int64_t(blockIdx.x + 1) * a.n_apply / n) != applied) apply_chunk(a, a.apply0 + applied);
  else sum_chunk(a, a.sum0 + int(blockIdx.x) - applied);
}

}  // namespace

struct mv_clip {
  int64_t n;                         // chunks
  int n_groups;
  int64_t longest;                   // elements of the longest group
  uintptr_t lo, hi;                  // addresses that the tensors span
  int n_tensors;
  struct Span { uintptr_t lo, hi; }* spans;      // host: the bytes of each tensor
  int empty;                         // some group has no chunk
  int n_stages;
  int32_t* stage;                    // host: [n_stages + 1] first chunk of each stage
  ClipArgs args;
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

int clip_launch(const ClipArgs& a, cudaStream_t st) {
  const unsigned grid = unsigned(a.n_apply + a.n_sum + a.empty);
  if (grid == 0) return MV_OK;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(TPB);
  cfg.stream = st;
  cudaLaunchAttribute early = {};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  const bool ok = cudaLaunchKernelEx(&cfg, k_clip, a) == cudaSuccess;
  return cuda_ok() == MV_OK && ok ? MV_OK : MV_ERR_CUDA;
}

// The norms only, or stage by stage: sum the first, then scale one while summing the next, then scale the last.
int clip_run(mv_clip* p, cudaStream_t st, float max_norm, float* rows, int64_t ld, float* norms, bool apply) {
  ClipArgs a = p->args;
  a.max_norm = max_norm; a.rows = rows; a.ld = ld; a.norms = norms;
  const int last = apply ? p->n_stages : 0;
  for (int s = 0; s <= last; ++s) {
    a.apply0 = s > 0 ? p->stage[s - 1] : 0;
    a.n_apply = s > 0 ? p->stage[s] - p->stage[s - 1] : 0;
    a.sum0 = s < p->n_stages ? p->stage[s] : 0;
    a.n_sum = s < p->n_stages ? p->stage[apply ? s + 1 : p->n_stages] - p->stage[s] : 0;
    a.empty = s == 0 && p->empty;
    if (int rc = clip_launch(a, st)) return rc;
  }
  return MV_OK;
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
  int32_t* stage = static_cast<int32_t*>(calloc(size_t(n_groups) + 1, 4));
  if (!p || !spans || !host || !stage) { free(p); free(spans); free(host); free(stage); return MV_ERR_WORKSPACE; }
  char* base = static_cast<char*>(workspace);
  p->n = L.n;
  p->n_groups = n_groups;
  p->n_tensors = n_tensors;
  p->spans = spans;
  p->lo = UINTPTR_MAX;
  p->stage = stage;
  p->args.chunks = reinterpret_cast<Chunk*>(base + L.chunks);
  p->args.first = reinterpret_cast<int32_t*>(base + L.first);
  p->args.ticket = reinterpret_cast<uint32_t*>(base + L.ticket);
  p->args.partial = reinterpret_cast<double*>(base + L.partial);
  p->args.coef = reinterpret_cast<float*>(base + L.coef);
  p->args.n_groups = n_groups;
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
  // stages: whole groups, as many as STAGE holds
  int64_t held = 0;
  for (g = 0; g < n_groups; ++g) {
    int64_t bytes = 0;
    for (int32_t k = first[g]; k < first[g + 1]; ++k) bytes += int64_t(c[k].n) * type_size(c[k].type);
    p->empty |= first[g] == first[g + 1];
    if (p->n_stages == 0 || (held > 0 && bytes > 0 && held + bytes > STAGE)) {
      stage[p->n_stages++] = first[g];
      held = 0;
    }
    held += bytes;
    stage[p->n_stages] = first[g + 1];
  }
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
  free(plan->stage);
  free(plan);
  return MV_OK;
}

int mv_clip_norm(mv_clip* plan, void* stream, float* norms) {
  if (!plan || !norms || misaligned(norms, 4)) return MV_ERR_INVALID_ARG;
  return clip_run(plan, static_cast<cudaStream_t>(stream), INFINITY, nullptr, 0, norms, false);
}

int mv_clip_scale(mv_clip* plan, void* stream, float max_norm, float* norms) {
  if (!plan || !(max_norm >= 0.0f) || misaligned(norms, 4)) return MV_ERR_INVALID_ARG;
  return clip_run(plan, static_cast<cudaStream_t>(stream), max_norm, nullptr, 0, norms, true);
}

int mv_clip_pack(mv_clip* plan, void* stream, float max_norm, float* rows, int64_t ld, float* norms) {
  if (!plan || !(max_norm >= 0.0f) || misaligned(norms, 4) || misaligned(rows, 4) || !rows || ld < plan->longest ||
      overlaps(plan, rows, ld))
    return MV_ERR_INVALID_ARG;
  return clip_run(plan, static_cast<cudaStream_t>(stream), max_norm, rows, ld, norms, true);
}

}  // extern "C"
