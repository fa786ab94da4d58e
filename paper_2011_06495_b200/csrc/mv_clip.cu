// mv_clip.cu -- norms over many tensors, one per group, and clipping in place or into the workers' rows, for sm_100a.
#include "mv_lm.cuh"

#include <algorithm>
#include <float.h>
#include <math.h>
#include <stdlib.h>

namespace {

// The list is cut into chunks of 32 KB, one CTA each.  A group's factor is known only when all its chunks have been summed.
// A short list, whose chunks all fit the shared memory of half the device, is read once: one kernel whose CTAs sum their
// chunk, keep it until the factor is there, and scale it.  A long one is read twice, by a kernel that sums and one that scales.
// Memory bounds both: ten groups of 11,173,962 fp32 are summed in 71 us (6.3 TB/s) and scaled into rows in 136 us (6.6 TB/s), or in place in 138.
// (Working a long list off group by group, so that the second reading finds its data in L2, gains nothing: L2 delivers hardly
// more than memory does, 8 to 9 TB/s against 7, and the stages' ends cost more: 232 to 274 us for the whole in four forms of it.)
constexpr int TPB = 256;
constexpr int CHUNK_BYTES = 32768;
constexpr int HOLD = 148 * 3;        // chunks of a short list: six fit a multiprocessor
constexpr int SPIN_LIMIT = 1 << 22;  // polls of a factor (a second or more) before a CTA gives up, unless the plan says otherwise

struct Chunk {
  void* ptr;                         // first element
  int64_t dst;                       // its place in the group's row
  int32_t n;
  int32_t type;
  int32_t group;
  int32_t pad;
};

inline int64_t chunk_len(int type) { return CHUNK_BYTES / type_size(type); }

struct Layout { size_t chunks, first, ticket, done, taken, gave_up, exact, partial, total; int64_t n; };

// types == nullptr: room for the longest list of chunks that any types give
inline bool clip_layout(const int64_t* numel, const int* types, int n_tensors, int n_groups, Layout* L) {
  if (n_tensors < 0 || (n_tensors > 0 && !numel) || n_groups < 1 || n_groups >= (1 << 20)) return false;
  L->n = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (numel[i] < 0 || numel[i] >= (int64_t(1) << 40)) return false;
    const int64_t len = chunk_len(types ? types[i] : MV_F32);
    L->n += (numel[i] + len - 1) / len;
  }
  if (L->n >= (int64_t(1) << 30)) return false;
  size_t o = 0;
  L->chunks = o;  o = align_up(o + size_t(L->n + 1) * sizeof(Chunk), 256);      // (an empty one more, for a list without elements)
  L->first = o;   o = align_up(o + size_t(n_groups + 1) * 4, 256);
  L->ticket = o;  o = align_up(o + size_t(n_groups) * 4, 256);
  L->done = o;    o = align_up(o + size_t(n_groups) * 8, 256);
  L->taken = o;   L->gave_up = o + 8;   o += 256;      // what the host fills ends here
  L->exact = o;   o = align_up(o + size_t(n_groups) * 8, 256);
  L->partial = o; o = align_up(o + size_t(L->n) * 8, 256);
  L->total = o;
  return true;
}

struct ClipArgs {
  const Chunk* chunks;
  const int32_t* first;              // [groups + 1] first chunk of each group
  uint32_t* ticket;                  // [groups] chunks summed so far; back to 0 with the last one
  unsigned long long* done;          // [groups] the factor's bits, and above them the number of the call that found it
  unsigned long long* taken;         // CTAs of the one-kernel form started so far, by all calls
  uint32_t* gave_up;                 // 1: a wait has run out since the host last asked
  double* exact;                     // [groups] the factor where 32 bits have no full precision for it
  double* partial;
  float* norms;
  float max_norm;
  float* rows;                       // pack: the rows; null: in place
  int64_t ld;
  int n_groups;
  int empty;                         // some group has no chunk
  int polls;                         // of a factor, before a CTA gives up
};

// 16 bytes of a chunk as numbers.
template <typename X> constexpr int PER = 16 / int(sizeof(X));
template <typename X> __device__ __forceinline__ void widen(const uint4& u, float (&f)[PER<X>]) {
  X x[PER<X>];
  memcpy(x, &u, 16);
#pragma unroll
  for (int i = 0; i < PER<X>; ++i) f[i] = to_f(x[i]);
}

// The parts of a chunk: its whole vectors, from the first 16-byte boundary on, and a single element e for a few threads.
template <typename X> struct Ends {
  int head, nv, e;
  float v;
  __device__ __forceinline__ Ends(const X* x, int n) {
    const int tid = threadIdx.x;
    head = min(n, int((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / int(sizeof(X)));
    nv = (n - head) / PER<X>;
    const int tail = head + nv * PER<X>;
    e = tid >= head + n - tail ? -1 : tid < head ? tid : tail + tid - head;
    v = e >= 0 ? to_f(x[e]) : 0.0f;
  }
};

// Squares of 16 bytes of numbers, added to two sums.  64 bits: a square of 32 bits has no room below 1e-19 or above 1e19.
template <typename X> __device__ __forceinline__ void add_squares(const uint4& u, double (&s)[2]) {
  float f[PER<X>];
  widen<X>(u, f);
#pragma unroll
  for (int j = 0; j < PER<X>; ++j) { const double v = f[j]; s[j & 1] = fma(v, v, s[j & 1]); }
}

// The norm and the factor of a group from its sum of squares.
__device__ __forceinline__ void put_norm(const ClipArgs& a, int g, double s, uint32_t call) {
  const double n = sqrt(s);
  if (a.norms) a.norms[g] = float(n);
  const double c = n > double(a.max_norm) && !isinf(n) ? double(a.max_norm) / n : 1.0;
  const float f = float(c);
  if (f < FLT_MIN) __stcg(a.exact + g, c);
  const unsigned long long w = (unsigned long long)call << 32 | __float_as_uint(f);
  asm volatile("st.release.gpu.u64 [%0], %1;" ::"l"(a.done + g), "l"(w) : "memory");
}

// A chunk's sum goes to its place, and the CTA that brings a group's last one adds them up, always in the same order.
__device__ __forceinline__ void finish_sum(const ClipArgs& a, int at, int group, double s, uint32_t call) {
  __shared__ double s_sum[TPB / 32];
  __shared__ int s_last;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int c0 = a.first[group], c1 = a.first[group + 1];
  auto together = [&] {              // over the CTA; the first thread has the result
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) s_sum[w] = s;
    __syncthreads();
    if (threadIdx.x == 0)
      for (int i = 1; i < TPB / 32; ++i) s += s_sum[i];
  };
  together();
  if (threadIdx.x == 0) {
    __stcg(a.partial + at, s);
    __threadfence();
    s_last = atomicAdd(a.ticket + group, 1u) == uint32_t(c1 - c0 - 1);
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  s = 0.0;
#pragma unroll 8
  for (int k = c0 + threadIdx.x; k < c1; k += TPB) s += __ldcg(a.partial + k);
  together();
  if (threadIdx.x == 0) {
    a.ticket[group] = 0;
    put_norm(a, group, s, call);
  }
}

template <typename X> struct alignas(4 * sizeof(X)) Four { X v[4]; };
template <typename X> __device__ __forceinline__ float4 times(const Four<X>& f, float c) {
  return make_float4(to_f(f.v[0]) * c, to_f(f.v[1]) * c, to_f(f.v[2]) * c, to_f(f.v[3]) * c);
}
template <typename X> __device__ __forceinline__ uint4 times(const uint4& u, float c) {
  float f[PER<X>];
  X y[PER<X>];
  widen<X>(u, f);
#pragma unroll
  for (int j = 0; j < PER<X>; ++j) y[j] = from_f<X>(f[j] * c);
  uint4 o;
  memcpy(&o, y, 16);
  return o;
}

// m elements from shared or global memory, times c, to 32 bits at dst.  Where the two do not lie alike, word by word, in whole
// aligned lines per warp: a sector written in two halves can cost a read.
template <typename X> __device__ __forceinline__ void pack(const X* from, int m, float c, float* dst) {
  const int tid = threadIdx.x;
  const int to16 = min(m, int((16 - (reinterpret_cast<uintptr_t>(dst) & 15)) & 15) / 4);
  if ((reinterpret_cast<uintptr_t>(from + to16) & (sizeof(Four<X>) - 1)) == 0) {
    const Four<X>* p = reinterpret_cast<const Four<X>*>(from + to16);
    float4* q = reinterpret_cast<float4*>(dst + to16);
    const int nf = (m - to16) / 4, tail = to16 + nf * 4;
    if (tid < to16 + m - tail) {
      const int e = tid < to16 ? tid : tail + tid - to16;
      dst[e] = to_f(from[e]) * c;
    }
#pragma unroll 1
    for (int i = tid; i < nf; i += 4 * TPB) {
      Four<X> f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + j * TPB < nf) f[j] = p[i + j * TPB];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + j * TPB < nf) __stcs(q + i + j * TPB, times(f[j], c));
    }
  } else {
    int i = tid - int(reinterpret_cast<uintptr_t>(dst) / 4 % 32);
    if (i >= 0 && i < m) dst[i] = to_f(from[i]) * c;
#pragma unroll 1
    for (i += TPB; i < m; i += 16 * TPB) {
      X f[16];
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (i + j * TPB < m) f[j] = from[i + j * TPB];
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (i + j * TPB < m) __stcs(dst + i + j * TPB, to_f(f[j]) * c);
    }
  }
}

// nv vectors times c, in place.
template <typename X> __device__ __forceinline__ void scale(const uint4* from, uint4* to, int nv, float c) {
#pragma unroll 1
  for (int i = threadIdx.x; i < nv; i += 4 * TPB) {
    uint4 u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j * TPB < nv) u[j] = from[i + j * TPB];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j * TPB < nv) __stcs(to + i + j * TPB, times<X>(u[j], c));
  }
}

// A chunk times a factor below the normal range of 32 bits (values near 1e38 clipped to a norm near 1): in 64 bits.  Seldom run.
template <typename X> __device__ __noinline__ void times_tiny(X* x, int n, double f, float* row) {
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += TPB) {
    const float y = float(double(to_f(x[i])) * f);
    if (row) row[i] = y;
    else x[i] = from_f<X>(y);
  }
}

// ------------------------------------------------------------------------------------------ a long list: two kernels
template <typename X> __device__ __forceinline__ double chunk_sum(const X* x, int n) {
  const Ends<X> ends(x, n);
  const uint4* p = reinterpret_cast<const uint4*>(x + ends.head) + threadIdx.x;
  const double single = ends.v;
  double s[2] = {single * single, 0.0};
#pragma unroll
  for (int i = 0; i < CHUNK_BYTES / 16 / TPB; i += 4) {
    uint4 u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = (i + j) * TPB + int(threadIdx.x) < ends.nv ? __ldg(p + (i + j) * TPB) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) add_squares<X>(u[j], s);
  }
  return s[0] + s[1];
}

__global__ void __launch_bounds__(TPB, 8) k_clip_sum(const __grid_constant__ ClipArgs a) {
  asm volatile("griddepcontrol.launch_dependents;");
  if (a.empty && blockIdx.x == 0)
    for (int g = threadIdx.x; g < a.n_groups; g += TPB)
      if (a.first[g] == a.first[g + 1]) put_norm(a, g, 0.0, 0);
  const Chunk c = a.chunks[blockIdx.x];
  if (c.n == 0) return;              // a list without elements
  const double s = c.type == MV_F32 ? chunk_sum(static_cast<const float*>(c.ptr), c.n)
                 : c.type == MV_BF16 ? chunk_sum(static_cast<const __nv_bfloat16*>(c.ptr), c.n)
                                     : chunk_sum(static_cast<const __half*>(c.ptr), c.n);
  finish_sum(a, blockIdx.x, c.group, s, 0);
}

template <typename X> __device__ __forceinline__ void chunk_scale(const ClipArgs& a, const Chunk& c, float f) {
  X* x = static_cast<X*>(c.ptr);
  if (f < FLT_MIN) {
    times_tiny<X>(x, c.n, __ldcg(a.exact + c.group), a.rows ? a.rows + c.group * a.ld + c.dst : nullptr);
  } else if (a.rows) {
    pack(static_cast<const X*>(x), c.n, f, a.rows + c.group * a.ld + c.dst);
  } else if (f != 1.0f) {
    const Ends<X> ends(x, c.n);
    if (ends.e >= 0) x[ends.e] = from_f<X>(ends.v * f);
    uint4* p = reinterpret_cast<uint4*>(x + ends.head);
    scale<X>(p, p, ends.nv, f);
  }
}

__global__ void __launch_bounds__(TPB, 5) k_clip_scale(const __grid_constant__ ClipArgs a) {
  const Chunk c = a.chunks[gridDim.x - 1 - blockIdx.x];      // backwards: the end of the list is what L2 still holds
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const float f = __uint_as_float(uint32_t(__ldcg(a.done + c.group)));
  if (c.type == MV_F32) chunk_scale<float>(a, c, f);
  else if (c.type == MV_BF16) chunk_scale<__nv_bfloat16>(a, c, f);
  else chunk_scale<__half>(a, c, f);
}

// ------------------------------------------------------------------------------------------ a short list: one kernel
// The group's factor, when it is there.  A NaN if it does not come in time (never expected): then what the CTA writes is NaN, and
// the host can ask for the word that says so.
__device__ __forceinline__ float wait_factor(const ClipArgs& a, int g, uint32_t call) {
  unsigned long long d = 0;
  for (int i = 0; i < a.polls; ++i) {
    asm volatile("ld.acquire.gpu.u64 %0, [%1];" : "=l"(d) : "l"(a.done + g) : "memory");
    if (uint32_t(d >> 32) == call) return __uint_as_float(uint32_t(d));
    __nanosleep(50);
  }
  *a.gave_up = 1;
  return __int_as_float(0x7fffffff);
}

template <typename X> __device__ __forceinline__ void sum_and_scale(const ClipArgs& a, const Chunk& c, uint32_t call, uint4* buf) {
  __shared__ float s_factor;
  X* x = static_cast<X*>(c.ptr);
  const Ends<X> ends(x, c.n);
  const uint4* p = reinterpret_cast<const uint4*>(x + ends.head);
#pragma unroll
  for (int i = threadIdx.x; i < CHUNK_BYTES / 16; i += TPB)
    if (i < ends.nv) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(uint32_t(__cvta_generic_to_shared(buf + i))), "l"(p + i) : "memory");
  const double single = ends.v;
  double s[2] = {single * single, 0.0};
  asm volatile("cp.async.wait_all;" ::: "memory");      // a thread sums the vectors that it fetched itself
#pragma unroll 2
  for (int i = threadIdx.x; i < ends.nv; i += TPB) add_squares<X>(buf[i], s);
  finish_sum(a, blockIdx.x, c.group, s[0] + s[1], call);
  if (threadIdx.x == 0) s_factor = wait_factor(a, c.group, call);
  __syncthreads();
  const float f = s_factor;
  if (f < FLT_MIN) {
    times_tiny<X>(x, c.n, __ldcg(a.exact + c.group), a.rows ? a.rows + c.group * a.ld + c.dst : nullptr);
  } else if (a.rows) {
    float* dst = a.rows + c.group * a.ld + c.dst;
    if (ends.e >= 0) dst[ends.e] = ends.v * f;
    pack(reinterpret_cast<const X*>(buf), ends.nv * PER<X>, f, dst + ends.head);
  } else if (f != 1.0f) {
    if (ends.e >= 0) x[ends.e] = from_f<X>(ends.v * f);
    scale<X>(buf, reinterpret_cast<uint4*>(x + ends.head), ends.nv, f);
  }
}

__global__ void __launch_bounds__(TPB, 6) k_clip_hold(const __grid_constant__ ClipArgs a) {
  __shared__ uint4 s_buf[CHUNK_BYTES / 16];
  __shared__ uint32_t s_call;
  if (threadIdx.x == 0) s_call = uint32_t(atomicAdd(a.taken, 1ull) / gridDim.x) + 1u;      // every call adds as many as it has CTAs
  const Chunk c = a.chunks[blockIdx.x];
  __syncthreads();
  if (a.empty && blockIdx.x == 0)
    for (int g = threadIdx.x; g < a.n_groups; g += TPB)
      if (a.first[g] == a.first[g + 1]) put_norm(a, g, 0.0, s_call);
  if (c.n == 0) return;              // a list without elements
  if (c.type == MV_F32) sum_and_scale<float>(a, c, s_call, s_buf);
  else if (c.type == MV_BF16) sum_and_scale<__nv_bfloat16>(a, c, s_call, s_buf);
  else sum_and_scale<__half>(a, c, s_call, s_buf);
}

}  // namespace

struct mv_clip {
  int64_t n;                         // chunks
  int hold;                          // chunks up to which the one-kernel form is used
  int n_groups;
  int64_t longest;                   // elements of the longest group
  uintptr_t lo, hi;                  // addresses that the tensors span
  int n_spans;
  struct Span { uintptr_t lo, hi; }* spans;      // host: the bytes of each tensor that has any, by address
  bool shared;                       // two of them share bytes
  ClipArgs args;
};

namespace {

// Whether the rows (of the longest group's length each) and one of the tensors share bytes.
bool overlaps(const mv_clip* p, const float* rows, int64_t ld) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(rows), hi = lo + (size_t(p->n_groups - 1) * ld + p->longest) * 4;
  if (hi <= p->lo || lo >= p->hi) return false;
  const uintptr_t pitch = uintptr_t(ld) * 4, len = uintptr_t(p->longest) * 4;
  for (int i = 0; i < p->n_spans; ++i) {
    const uintptr_t a = p->spans[i].lo, b = p->spans[i].hi;
    if (a >= hi || b <= lo) continue;
    if (a <= lo) return true;
    const uintptr_t row = lo + (a - lo) / pitch * pitch;      // the last one that begins at the tensor or before it
    if (a < row + len || b > row + pitch) return true;        // (in a gap, so another row follows)
  }
  return false;
}

int clip_run(mv_clip* p, cudaStream_t st, float max_norm, float* rows, int64_t ld, float* norms, bool apply) {
  ClipArgs a = p->args;
  a.max_norm = max_norm; a.rows = rows; a.ld = ld; a.norms = norms;
  const unsigned grid = unsigned(p->n > 0 ? p->n : 1);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(TPB);
  cfg.stream = st;
  cudaLaunchAttribute attr = {};
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  bool ok;
  if (apply && p->n <= p->hold) {
    attr.id = cudaLaunchAttributeCooperative;        // all CTAs at once or none: they wait for one another
    attr.val.cooperative = 1;
    ok = cudaLaunchKernelEx(&cfg, k_clip_hold, a) == cudaSuccess;
  } else {
    k_clip_sum<<<grid, TPB, 0, st>>>(a);
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    ok = !apply || cudaLaunchKernelEx(&cfg, k_clip_scale, a) == cudaSuccess;
  }
  return cuda_ok() == MV_OK && ok ? MV_OK : MV_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t mv_clip_workspace_bytes(const int64_t* numel, int n_tensors, int n_groups) {
  Layout L;
  return clip_layout(numel, nullptr, n_tensors, n_groups, &L) ? L.total : 0;
}

int mv_clip_create(mv_clip** out, void* stream, void* const* tensors, const int* types, const int64_t* numel, const int* groups,
                   int n_tensors, int n_groups, void* workspace, size_t workspace_bytes) {
  Layout L;
  if (!out || (n_tensors > 0 && (!tensors || !types)) || misaligned(workspace, 256) || !clip_layout(numel, nullptr, n_tensors, n_groups, &L))
    return MV_ERR_INVALID_ARG;
  const size_t need = L.total;
  for (int i = 0; i < n_tensors; ++i) {
    const int g = groups ? groups[i] : 0;
    if (!is_value_type(types[i]) || (numel[i] > 0 && !tensors[i]) || misaligned(tensors[i], type_size(types[i])) || g < 0 || g >= n_groups ||
        (i > 0 && groups && g < groups[i - 1]))
      return MV_ERR_INVALID_ARG;
  }
  if (!workspace || workspace_bytes < need) return MV_ERR_WORKSPACE;
  clip_layout(numel, types, n_tensors, n_groups, &L);
  mv_clip* p = static_cast<mv_clip*>(calloc(1, sizeof(mv_clip)));
  mv_clip::Span* spans = static_cast<mv_clip::Span*>(calloc(n_tensors ? n_tensors : 1, sizeof(mv_clip::Span)));
  char* host = static_cast<char*>(calloc(1, L.exact));
  if (!p || !spans || !host) { free(p); free(spans); free(host); return MV_ERR_WORKSPACE; }
  char* base = static_cast<char*>(workspace);
  p->n = L.n;
  p->n_groups = n_groups;
  p->spans = spans;
  p->lo = UINTPTR_MAX;
  p->args.chunks = reinterpret_cast<Chunk*>(base + L.chunks);
  p->args.first = reinterpret_cast<int32_t*>(base + L.first);
  p->args.ticket = reinterpret_cast<uint32_t*>(base + L.ticket);
  p->args.done = reinterpret_cast<unsigned long long*>(base + L.done);
  p->args.taken = reinterpret_cast<unsigned long long*>(base + L.taken);
  p->args.gave_up = reinterpret_cast<uint32_t*>(base + L.gave_up);
  p->args.exact = reinterpret_cast<double*>(base + L.exact);
  p->args.partial = reinterpret_cast<double*>(base + L.partial);
  p->args.polls = SPIN_LIMIT;
  p->args.n_groups = n_groups;
  Chunk* c = reinterpret_cast<Chunk*>(host + L.chunks);
  int32_t* first = reinterpret_cast<int32_t*>(host + L.first);
  int64_t nc = 0, dst = 0;
  int g = 0;
  first[0] = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const int gi = groups ? groups[i] : 0;
    while (g < gi) { first[++g] = int32_t(nc); dst = 0; }
    const int64_t len = chunk_len(types[i]);
    for (int64_t o = 0; o < numel[i]; o += len, ++nc) {
      c[nc].ptr = static_cast<char*>(tensors[i]) + o * type_size(types[i]);
      c[nc].dst = dst + o;
      c[nc].n = int32_t(numel[i] - o < len ? numel[i] - o : len);
      c[nc].type = types[i];
      c[nc].group = gi;
    }
    if (numel[i] > 0) {
      const uintptr_t lo = reinterpret_cast<uintptr_t>(tensors[i]), hi = lo + size_t(numel[i]) * type_size(types[i]);
      spans[p->n_spans++] = {lo, hi};
      p->lo = lo < p->lo ? lo : p->lo;
      p->hi = hi > p->hi ? hi : p->hi;
    }
    dst += numel[i];
    if (dst > p->longest) p->longest = dst;
  }
  while (g < n_groups) first[++g] = int32_t(nc);
  for (g = 0; g < n_groups; ++g) p->args.empty |= first[g] == first[g + 1];
  std::sort(spans, spans + p->n_spans, [](const mv_clip::Span& a, const mv_clip::Span& b) { return a.lo < b.lo; });
  for (int i = 1; i < p->n_spans; ++i) p->shared |= spans[i].lo < spans[i - 1].hi;
  // the one-kernel form needs all its CTAs at once
  int dev = 0, sms = 0, per_sm = 0;
  if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess &&
      cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, k_clip_hold, TPB, 0) == cudaSuccess)
    p->hold = sms * per_sm / 2 < HOLD ? sms * per_sm / 2 : HOLD;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool ok = cudaMemcpyAsync(base, host, L.exact, cudaMemcpyHostToDevice, st) == cudaSuccess && cudaStreamSynchronize(st) == cudaSuccess;
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

int mv_clip_status(mv_clip* plan, void* stream) {
  if (!plan) return MV_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  uint32_t flag = 0;
  if (cudaMemcpyAsync(&flag, plan->args.gave_up, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaMemsetAsync(plan->args.gave_up, 0, 4, st) != cudaSuccess ||
      cudaStreamSynchronize(st) != cudaSuccess) {
    cudaGetLastError();
    return MV_ERR_CUDA;
  }
  return flag ? MV_ERR_TIMEOUT : MV_OK;
}

int mv_clip_set_polls(mv_clip* plan, int polls) {
  if (!plan || polls < -1) return MV_ERR_INVALID_ARG;
  plan->args.polls = polls < 0 ? SPIN_LIMIT : polls;
  return MV_OK;
}

int mv_clip_norm(mv_clip* plan, void* stream, float* norms) {
  if (!plan || !norms || misaligned(norms, 4)) return MV_ERR_INVALID_ARG;
  return clip_run(plan, static_cast<cudaStream_t>(stream), INFINITY, nullptr, 0, norms, false);
}

int mv_clip_scale(mv_clip* plan, void* stream, float max_norm, float* norms) {
  if (!plan || plan->shared || !(max_norm >= 0.0f) || misaligned(norms, 4)) return MV_ERR_INVALID_ARG;
  return clip_run(plan, static_cast<cudaStream_t>(stream), max_norm, nullptr, 0, norms, true);
}

int mv_clip_pack(mv_clip* plan, void* stream, float max_norm, float* rows, int64_t ld, float* norms) {
  if (!plan || !(max_norm >= 0.0f) || misaligned(norms, 4) || misaligned(rows, 4) || !rows || ld < plan->longest ||
      overlaps(plan, rows, ld))
    return MV_ERR_INVALID_ARG;
  return clip_run(plan, static_cast<cudaStream_t>(stream), max_norm, rows, ld, norms, true);
}

}  // extern "C"
