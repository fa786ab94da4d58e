// mv_embed.cu -- embedding lookup with scaling, and its gradient by sorted tokens, for sm_100a.
#include "mv_lm.cuh"

namespace {

// ------------------------------------------------------------------------------------------ lookup
template <typename W, typename O>
__global__ void __launch_bounds__(256) k_embed(const W* __restrict__ weight, int64_t V, int64_t D, int64_t ldw, const void* __restrict__ ids,
                                                int id_type, int64_t T, float scale, O* __restrict__ out, int64_t ldo) {
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    const int64_t v = load_id(ids, id_type, t, V);
    for (int64_t j = threadIdx.x; j < D; j += blockDim.x)
      out[t * ldo + j] = v >= 0 ? from_f<O>(to_f(weight[v * ldw + j]) * scale) : from_f<O>(0.0f);
  }
}

// ------------------------------------------------------------------------------------------ gradient
// The tokens fall into `nb` buckets (a power of two) by id mod nb, so that the frequent tokens, which have
// neighbouring ids, spread over all buckets.  The CTA of a bucket reads all ids, counts its own ids in shared
// memory (one counter per id / nb) and writes its tokens grouped by id, in token order, to `perm`.
constexpr int SORT_TPB = 256;
constexpr int SORT_BINS = 8192;      // ids per bucket, at most

struct EmbedWs { size_t perm, row, total; };
inline EmbedWs embed_ws(int64_t T) {
  EmbedWs L;
  size_t o = 0;
  L.perm = o; o = align_up(o + size_t(T) * 4, 16);
  L.row = o;  o = align_up(o + size_t(T) * 4, 16);
  L.total = o ? o : 16;
  return L;
}

inline int64_t bucket_count(int64_t V) {
  int64_t nb = 128;
  while ((V + nb - 1) / nb > SORT_BINS) nb *= 2;
  return nb;
}

__global__ void __launch_bounds__(SORT_TPB) k_embed_sort(const void* __restrict__ ids, int id_type, int64_t T, int64_t V, int64_t pad_id,
                                                          int nb_log, int32_t* __restrict__ perm, int32_t* __restrict__ row) {
  extern __shared__ uint32_t cnt[];                 // [ids of this bucket]: tokens per id, then the next slot of the id
  __shared__ uint32_t s_below, s_scan[SORT_TPB];
  const int64_t nb = int64_t(1) << nb_log;
  const int b = blockIdx.x;
  const int bins = int((V - b + nb - 1) >> nb_log);
  for (int i = threadIdx.x; i < bins; i += SORT_TPB) cnt[i] = 0;
  if (threadIdx.x == 0) s_below = 0;
  __syncthreads();
  uint32_t below = 0;
  for (int64_t t = threadIdx.x; t < T; t += SORT_TPB) {
    const int64_t v = load_id(ids, id_type, t, V);
    if (v < 0 || v == pad_id) continue;
    const int64_t m = v & (nb - 1);
    if (m < b) ++below;
    else if (m == b) atomicAdd(&cnt[v >> nb_log], 1u);
  }
  atomicAdd(&s_below, below);
  __syncthreads();
  // exclusive scan of the counters: every thread takes consecutive ones
  const int per = (bins + SORT_TPB - 1) / SORT_TPB;
  const int i0 = min(bins, int(threadIdx.x) * per), i1 = min(bins, i0 + per);
  uint32_t sum = 0;
  for (int i = i0; i < i1; ++i) sum += cnt[i];
  s_scan[threadIdx.x] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t run = s_below;
    for (int i = 0; i < SORT_TPB; ++i) { uint32_t c = s_scan[i]; s_scan[i] = run; run += c; }
  }
  __syncthreads();
  uint32_t run = s_scan[threadIdx.x];
  for (int i = i0; i < i1; ++i) { uint32_t c = cnt[i]; cnt[i] = run; run += c; }
  __syncthreads();
  // the first warp goes through the tokens in order
  if (threadIdx.x >= 32) return;
  for (int64_t t0 = 0; t0 < T; t0 += 32) {
    const int64_t t = t0 + threadIdx.x;
    const int64_t v = t < T ? load_id(ids, id_type, t, V) : -1;
    const bool mine = v >= 0 && v != pad_id && (v & (nb - 1)) == b;
    const unsigned any = __ballot_sync(0xffffffffu, mine);
    if (!any) continue;
    if (mine) {
      const unsigned same = __match_any_sync(any, int(v));
      const int rank = __popc(same & ((1u << threadIdx.x) - 1u));
      const uint32_t slot = cnt[v >> nb_log] + rank;
      perm[slot] = int32_t(t);
      row[slot] = int32_t(v);
      __syncwarp(any);
      if (rank == 0) cnt[v >> nb_log] += __popc(same);
    }
    __syncwarp();
  }
}

__global__ void k_zero(float* __restrict__ dst, int64_t V, int64_t D, int64_t ldw) {
  for (int64_t v = blockIdx.x; v < V; v += gridDim.x)
    for (int64_t j = threadIdx.x; j < D; j += blockDim.x) dst[v * ldw + j] = 0.0f;
}

// A CTA per sorted position; the one that starts a run sums it.
template <typename T_>
__global__ void __launch_bounds__(256) k_embed_sum(const T_* __restrict__ dout, int64_t ldd, const int32_t* __restrict__ perm, const int32_t* __restrict__ row,
                                                    int64_t T, int64_t D, float scale, int accumulate, float* __restrict__ dweight, int64_t ldw) {
  for (int64_t s = blockIdx.x; s < T; s += gridDim.x) {
    const int32_t v = row[s];
    if (v < 0 || (s > 0 && row[s - 1] == v)) continue;
    for (int64_t j = threadIdx.x; j < D; j += blockDim.x) {
      float acc = 0.0f;
      for (int64_t u = s; u < T && row[u] == v; ++u) acc += to_f(dout[int64_t(perm[u]) * ldd + j]);
      float* p = dweight + int64_t(v) * ldw + j;
      *p = accumulate ? *p + acc * scale : acc * scale;
    }
  }
}

}  // namespace

extern "C" {

int mv_embed(void* stream, const void* weight, int w_type, int64_t V, int64_t D, int64_t ldw, const void* ids, int id_type,
             int64_t T, float scale, void* out, int out_type, int64_t ldo) {
  const int64_t lim = int64_t(1) << 31;
  if (!is_value_type(w_type) || !is_value_type(out_type) || !is_id_type(id_type) || V < 1 || V >= lim || D < 1 || D >= lim || T < 0 ||
      T >= lim || ldw < D || ldo < D || !weight || (T > 0 && (!ids || !out)) || misaligned(weight, type_size(w_type)) ||
      misaligned(ids, type_size(id_type)) || misaligned(out, type_size(out_type)))
    return MV_ERR_INVALID_ARG;
  if (T == 0) return MV_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_type(w_type, [&](auto w) {
    return with_type(out_type, [&](auto o) {
      using W = decltype(w);
      using O = decltype(o);
      k_embed<W, O><<<unsigned(T < (1 << 16) ? T : (1 << 16)), 256, 0, st>>>(static_cast<const W*>(weight), V, D, ldw, ids, id_type, T, scale,
                                                                              static_cast<O*>(out), ldo);
      return cuda_ok();
    });
  });
}

size_t mv_embed_grad_workspace_bytes(int64_t T, int64_t V, int64_t D) {
  const int64_t lim = int64_t(1) << 31;
  if (T < 0 || T >= lim || V < 1 || V >= lim || D < 1 || D >= lim) return 0;
  return embed_ws(T).total;
}

int mv_embed_grad(void* stream, const void* dout, int dout_type, int64_t ldd, const void* ids, int id_type, int64_t T, int64_t V,
                  int64_t D, float scale, int64_t pad_id, int accumulate, float* dweight, int64_t ldw, void* workspace,
                  size_t workspace_bytes) {
  const int64_t lim = int64_t(1) << 31;
  if (!is_value_type(dout_type) || !is_id_type(id_type) || T < 0 || T >= lim || V < 1 || V >= lim || D < 1 || D >= lim || ldd < D ||
      ldw < D || (accumulate != 0 && accumulate != 1) || !dweight || (T > 0 && (!dout || !ids)) || misaligned(dout, type_size(dout_type)) ||
      misaligned(ids, type_size(id_type)) || misaligned(dweight, 4) || misaligned(workspace, 16))
    return MV_ERR_INVALID_ARG;
  const EmbedWs L = embed_ws(T);
  if (!workspace || workspace_bytes < L.total) return MV_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t* perm = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + L.perm);
  int32_t* row = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + L.row);
  if (!accumulate) k_zero<<<unsigned(V < (1 << 16) ? V : (1 << 16)), 256, 0, st>>>(dweight, V, D, ldw);
  if (T == 0) return cuda_ok();
  if (cudaMemsetAsync(row, 0xff, size_t(T) * 4, st) != cudaSuccess) return MV_ERR_CUDA;
  const int64_t nb = bucket_count(V);
  int nb_log = 0;
  while ((int64_t(1) << nb_log) < nb) ++nb_log;
  const int64_t buckets = V < nb ? V : nb;
  const size_t smem = size_t((V + nb - 1) / nb) * 4;
  k_embed_sort<<<unsigned(buckets), SORT_TPB, smem, st>>>(ids, id_type, T, V, pad_id, nb_log, perm, row);
  return with_type(dout_type, [&](auto x) {
    using X = decltype(x);
    k_embed_sum<X><<<unsigned(T < (1 << 16) ? T : (1 << 16)), 256, 0, st>>>(static_cast<const X*>(dout), ldd, perm, row, T, D, scale, accumulate,
                                                                             dweight, ldw);
    return cuda_ok();
  });
}

}  // extern "C"
