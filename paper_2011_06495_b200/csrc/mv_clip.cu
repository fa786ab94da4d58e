// mv_clip.cu -- norms over many tensors, one per group, and clipping in place or into the workers' rows, for sm_100a.
#include "mv_lm.cuh"

#include <math.h>
#include <stdlib.h>

namespace {

// The list is cut into chunks.  A group's factor is known only when all its chunks have been summed, so every element is
// read twice; to read it from memory only once, the list is worked off in stages of whole groups that fit L2.  One kernel does
// all of it, one CTA per item (sum this chunk, scale that chunk), in the order: the sums of stage 0, then the scalings
// of stage s mixed with the sums of stage s + 1.  CTAs take their items by a counter, so an item's predecessors are with CTAs
// that run or have run; an item that scales waits for its group's factor, and the sums that it waits for wait for nothing.
// The last HOLD chunks of a group (all of a small group) are read only once: their CTAs sum them, keep them in shared memory
// until the factor is there, and scale them.  Half of the device's CTAs are enough for that, so they cannot wait in vain.
constexpr int TPB = 256;
constexpr int CHUNK = 8192;          // elements per chunk: 16 or 32 KB, all on their way at once, six chunks a multiprocessor
constexpr int LEAD = 148 * 6;        // sums of the next stage taken before the first scaling: its factors are there by then
#ifndef HOLDN
#define HOLDN 3
#endif
constexpr int HOLD = 148 * HOLDN;
constexpr int SPIN_LIMIT = 1 << 22;  // polls of a factor (a second or more) before an item is given up

struct Chunk {
  void* ptr;                         // first element
  int64_t dst;                       // its place in the group's row
  int32_t n;
  int32_t type;
  int32_t group;
  int32_t what;                      // 4 x the chunk's number + SUM, SCALE or both
};

enum { SUM = 1, SCALE = 2 };

struct Layout { size_t sums, items, first, ticket, done, taken, partial, total; int64_t n; };

inline bool clip_layout(const int64_t* numel, int n_tensors, int n_groups, Layout* L) {
  if (n_tensors < 0 || (n_tensors > 0 && !numel) || n_groups < 1 || n_groups >= (1 << 20)) return false;
  L->n = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (numel[i] < 0 || numel[i] >= (int64_t(1) << 40)) return false;
    L->n += (numel[i] + CHUNK - 1) / CHUNK;
  }
  if (L->n >= (int64_t(1) << 29)) return false;
  size_t o = 0;
  L->sums = o;    o = align_up(o + size_t(L->n + 1) * sizeof(Chunk), 256);      // (an empty one more, for a list without elements)
  L->items = o;   o = align_up(o + size_t(L->n + 1) * 2 * sizeof(Chunk), 256);
  L->first = o;   o = align_up(o + size_t(n_groups + 1) * 4, 256);
  L->ticket = o;  o = align_up(o + size_t(n_groups) * 4, 256);
  L->done = o;    o = align_up(o + size_t(n_groups) * 8, 256);
  L->taken = o;   o += 256;          // what the host fills ends here
  L->partial = o; o = align_up(o + size_t(L->n) * 8, 256);
  L->total = o;
  return true;
}

struct ClipArgs {
  const Chunk* items;
  unsigned long long* taken;         // items taken so far, by all calls of this kind
  const int32_t* first;              // [groups + 1] first chunk of each group
  uint32_t* ticket;                  // [groups] chunks summed so far; back to 0 with the last one
  unsigned long long* done;          // [groups] number of the scaling call (from 1) and the factor's bits, once it is known
  double* partial;
  float* norms;
  float max_norm;
  float* rows;                       // pack: the rows; null: in place
  int64_t ld;
  int n_groups;
  int empty;                         // some group has no chunk
  int scales;                        // 0: a call for the norms alone
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

// The chunk's whole vectors on their way to shared memory, vector i * TPB + thread at that place.
template <typename X> __device__ __forceinline__ void fetch(const X* x, int nv, uint4* buf) {
  constexpr int V = CHUNK / PER<X> / TPB;
  const uint4* p = reinterpret_cast<const uint4*>(x) + threadIdx.x;
  const uint32_t to = uint32_t(__cvta_generic_to_shared(buf + threadIdx.x));
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i * TPB + int(threadIdx.x) < nv)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + i * TPB * 16), "l"(p + i * TPB) : "memory");
}

// Sum of squares of a chunk in shared memory, this thread's part.  64 bits: a square of 32 bits has no room below 1e-19 or
// above 1e19.
template <typename X> __device__ __forceinline__ double chunk_sum(int nv, const uint4* buf, double single) {
  double s = single * single;
#pragma unroll 2
  for (int i = threadIdx.x; i < nv; i += TPB) {
    float f[PER<X>];
    widen<X>(buf[i], f);
#pragma unroll
    for (int j = 0; j < PER<X>; ++j) { const double v = f[j]; s = fma(v, v, s); }
  }
  return s;
}

// The norm and the factor of a group from its sum of squares.
__device__ __forceinline__ void put_norm(const ClipArgs& a, int g, double s, uint32_t call) {
  const double n = sqrt(s);
  if (a.norms) a.norms[g] = float(n);
  const float f = n > double(a.max_norm) && !isinf(n) ? float(double(a.max_norm) / n) : 1.0f;
  const unsigned long long w = (unsigned long long)call << 32 | __float_as_uint(f);
  asm volatile("st.release.gpu.u64 [%0], %1;" ::"l"(a.done + g), "l"(w) : "memory");
}

// The first warp: a chunk's sum goes to its place, and the CTA that brings a group's last one adds them up, always in the
// same order.
__device__ __forceinline__ void finish_sum(const ClipArgs& a, const Chunk& c, double s, uint32_t call) {
  const int lane = threadIdx.x, c0 = a.first[c.group], c1 = a.first[c.group + 1];
  uint32_t arrived = 0;
  if (lane == 0) {
    __stcg(a.partial + (c.what >> 2), s);
    __threadfence();
    arrived = atomicAdd(a.ticket + c.group, 1u);
  }
  if (__shfl_sync(0xffffffffu, arrived, 0) != uint32_t(c1 - c0 - 1)) return;
  __threadfence();
  s = 0.0;
#pragma unroll 8
  for (int k = c0 + lane; k < c1; k += 32) s += __ldcg(a.partial + k);
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) {
    a.ticket[c.group] = 0;
    put_norm(a, c.group, s, call);
  }
}

// The group's factor, when it is there.  A NaN if it does not come in time (never expected): what the item writes is NaN.
__device__ __forceinline__ float wait_factor(const ClipArgs& a, int g, uint32_t call) {
  unsigned long long d = 0;
  for (int i = 0; i < SPIN_LIMIT; ++i) {
    asm volatile("ld.acquire.gpu.u64 %0, [%1];" : "=l"(d) : "l"(a.done + g) : "memory");
    if (uint32_t(d >> 32) == call) return __uint_as_float(uint32_t(d));
    __nanosleep(50);
  }
  return __int_as_float(0x7fffffff);
}

// A chunk in shared memory times its group's factor: in place, or to 32 bits at dst.
template <typename X> __device__ __forceinline__ void chunk_scale(X* x, float* dst, int head, int nv, int e, float v, const uint4* buf, float c) {
  const int tid = threadIdx.x;
  if (dst) {
    if (e >= 0) dst[e] = v * c;
    dst += head;
    const int m = nv * PER<X>;
    if ((reinterpret_cast<uintptr_t>(dst) & 15) == 0) {
      struct alignas(4 * sizeof(X)) Four { X v[4]; };
      const Four* from = reinterpret_cast<const Four*>(buf);
#pragma unroll 4
      for (int i = tid; i < m / 4; i += TPB) {
        const Four f = from[i];
        __stcs(reinterpret_cast<float4*>(dst) + i, make_float4(to_f(f.v[0]) * c, to_f(f.v[1]) * c, to_f(f.v[2]) * c, to_f(f.v[3]) * c));
      }
    } else {                         // word by word, whole aligned lines per warp (sectors written in two halves cost a read each)
      const X* from = reinterpret_cast<const X*>(buf);
      const int i0 = tid - int(reinterpret_cast<uintptr_t>(dst) / 4 % 32);
      if (i0 >= 0 && i0 < m) __stcs(dst + i0, to_f(from[i0]) * c);
#pragma unroll 8
      for (int i = i0 + TPB; i < m; i += TPB) __stcs(dst + i, to_f(from[i]) * c);
    }
  } else if (c != 1.0f) {
    if (e >= 0) x[e] = from_f<X>(v * c);
    uint4* p = reinterpret_cast<uint4*>(x + head);
#pragma unroll 2
    for (int i = tid; i < nv; i += TPB) {
      float f[PER<X>];
      X y[PER<X>];
      widen<X>(buf[i], f);
#pragma unroll
      for (int j = 0; j < PER<X>; ++j) y[j] = from_f<X>(f[j] * c);
      uint4 o;
      memcpy(&o, y, 16);
      __stcs(p + i, o);
    }
  }
}

template <typename X> __device__ __forceinline__ void work_off(const ClipArgs& a, const Chunk& c, uint32_t call, uint4* buf) {
  __shared__ double s_sum[TPB / 32];
  __shared__ float s_factor;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, tid = threadIdx.x, n = c.n;
  X* x = static_cast<X*>(c.ptr);
  const int head = head_of(x, n), nv = (n - head) / PER<X>, tail = head + nv * PER<X>;
  fetch(x + head, nv, buf);
  // what lies before and behind the whole vectors: an element e for a few threads
  const int e = tid >= head + n - tail ? -1 : tid < head ? tid : tail + tid - head;
  const float v = e >= 0 ? to_f(x[e]) : 0.0f;
  if (c.what & SUM) {
    asm volatile("cp.async.wait_all;" ::: "memory");      // a thread sums the vectors that it fetched itself
    double s = chunk_sum<X>(nv, buf, v);
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) s_sum[w] = s;
    __syncthreads();
    if (w == 0) {
      s = lane < TPB / 32 ? s_sum[lane] : 0.0;
      for (int o = TPB / 64; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      finish_sum(a, c, s, call);
    }
  }
  if (!(c.what & SCALE)) return;
  if (tid == TPB - 1) s_factor = wait_factor(a, c.group, call);
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  chunk_scale(x, a.rows ? a.rows + c.group * a.ld + c.dst : nullptr, head, nv, e, v, buf, s_factor);
}

__global__ void __launch_bounds__(TPB, 6) k_clip(const __grid_constant__ ClipArgs a) {
  __shared__ uint4 s_buf[CHUNK * 4 / 16];
  __shared__ unsigned long long s_at;
  if (threadIdx.x == 0) s_at = atomicAdd(a.taken, 1ull);
  __syncthreads();
  // every call takes as many items as it has CTAs: the remainder is the item, the quotient the call
  const uint32_t at = uint32_t(s_at % gridDim.x), call = a.scales ? uint32_t(s_at / gridDim.x) + 1u : 0u;
  if (a.empty && at == 0)
    for (int g = threadIdx.x; g < a.n_groups; g += TPB)
      if (a.first[g] == a.first[g + 1]) put_norm(a, g, 0.0, call);
  const Chunk c = a.items[at];
  if (c.type == MV_F32) work_off<float>(a, c, call, s_buf);
  else if (c.type == MV_BF16) work_off<__nv_bfloat16>(a, c, call, s_buf);
  else work_off<__half>(a, c, call, s_buf);
}

}  // namespace

struct mv_clip {
  int64_t n;                         // chunks
  int n_groups;
  int64_t longest;                   // elements of the longest group
  uintptr_t lo, hi;                  // addresses that the tensors span
  int n_tensors;
  struct Span { uintptr_t lo, hi; }* spans;      // host: the bytes of each tensor
  const Chunk *sums, *items;         // the sums alone, and sums and scalings in their order
  int64_t n_items;
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

int clip_run(mv_clip* p, cudaStream_t st, float max_norm, float* rows, int64_t ld, float* norms, bool apply) {
  ClipArgs a = p->args;
  a.max_norm = max_norm; a.rows = rows; a.ld = ld; a.norms = norms;
  a.items = apply ? p->items : p->sums;
  a.scales = apply;
  a.taken += apply ? 1 : 0;          // the two kinds of call count their items apart
  const int64_t n = apply ? p->n_items : p->n;
  k_clip<<<unsigned(n > 0 ? n : 1), TPB, 0, st>>>(a);
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
  p->sums = reinterpret_cast<Chunk*>(base + L.sums);
  p->items = reinterpret_cast<Chunk*>(base + L.items);
  p->args.first = reinterpret_cast<int32_t*>(base + L.first);
  p->args.ticket = reinterpret_cast<uint32_t*>(base + L.ticket);
  p->args.done = reinterpret_cast<unsigned long long*>(base + L.done);
  p->args.taken = reinterpret_cast<unsigned long long*>(base + L.taken);
  p->args.partial = reinterpret_cast<double*>(base + L.partial);
  p->args.n_groups = n_groups;
  Chunk* c = reinterpret_cast<Chunk*>(host + L.sums);
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
      c[nc].what = int32_t(4 * nc + SUM);
    }
    spans[i].lo = reinterpret_cast<uintptr_t>(tensors[i]);
    spans[i].hi = spans[i].lo + size_t(numel[i]) * type_size(types[i]);
    if (numel[i] > 0 && spans[i].lo < p->lo) p->lo = spans[i].lo;
    if (numel[i] > 0 && spans[i].hi > p->hi) p->hi = spans[i].hi;
    dst += numel[i];
    if (dst > p->longest) p->longest = dst;
  }
  while (g < n_groups) first[++g] = int32_t(nc);
  // Items of a call that scales.  A group's own: the sums of all but its last HOLD chunks, then those in one go.  Then the
  // scalings of the former, mixed with the next group's own items.
  Chunk* item = reinterpret_cast<Chunk*>(host + L.items);
  int64_t z0 = 0, z1 = 0;            // chunks still to be scaled
  for (g = 0; g <= n_groups; ++g) {
    const int64_t f0 = g < n_groups ? first[g] : 0, f1 = g < n_groups ? first[g + 1] : 0;
    if (g < n_groups) p->args.empty |= f0 == f1;
    if (g < n_groups && f0 == f1) continue;
    const int64_t own = f1 - f0, held = own < HOLD ? own : HOLD, nz = z1 - z0, lead = own < LEAD ? own : LEAD;
    for (int64_t i = 0, oi = 0, zi = 0; i < own + nz; ++i) {
      if (i < lead || (i + 1 - lead) * nz / (own + nz - lead) <= zi) {
        *item = c[f0 + oi++];
        if (oi > own - held) item->what |= SCALE;
      } else {
        *item = c[z0 + zi++];
        item->what ^= SUM | SCALE;
      }
      ++item;
    }
    z0 = f0;
    z1 = f1 - held;
  }
  p->n_items = item - reinterpret_cast<Chunk*>(host + L.items);
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
