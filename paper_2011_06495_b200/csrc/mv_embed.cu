// mv_embed.cu -- embedding lookup with scaling, and its gradient by sorted tokens, for sm_100a.
//
// Both only move bytes (a multiplication or an addition per element), so both are bound by memory: what counts is
// that every lane has several independent 16-byte loads in flight and that nothing is moved twice.
#include "mv_lm.cuh"

namespace {

// A lane's share of a row: 16 bytes of the input type where the rows allow it (VEC: consecutive elements), else as many
// single elements, 32 apart, so that a warp's accesses stay contiguous.
template <typename X> constexpr int LANE = 16 / int(sizeof(X));
template <typename X> constexpr int BLOCK = 32 * LANE<X>;         // columns per warp

template <typename X, bool VEC> __device__ __forceinline__ int64_t column(int64_t cb, int lane, int j, int lanes = 32) {
  return VEC ? cb * BLOCK<X> + lane * LANE<X> + j : cb * BLOCK<X> + j * lanes + lane;
}

// The raw elements of one row, loaded without being converted (so that loads of several rows can be outstanding).
template <typename X> struct Raw { X e[LANE<X>]; };

template <typename X, bool VEC> __device__ __forceinline__ void load_raw(const X* row, int64_t D, int64_t cb, int lane, int lanes, uint4& u) {
  Raw<X> r;
  if constexpr (VEC) {
    const int64_t c0 = column<X, true>(cb, lane, 0);
    if (c0 + LANE<X> <= D) {
      u = __ldg(reinterpret_cast<const uint4*>(row + c0));
      return;
    }
#pragma unroll
    for (int j = 0; j < LANE<X>; ++j) r.e[j] = c0 + j < D ? row[c0 + j] : from_f<X>(0.0f);
  } else {
#pragma unroll
    for (int j = 0; j < LANE<X>; ++j) {
      const int64_t c = column<X, false>(cb, lane, j, lanes);
      r.e[j] = c < D ? row[c] : from_f<X>(0.0f);
    }
  }
  memcpy(&u, &r, 16);
}

// ------------------------------------------------------------------------------------------ lookup
// A warp takes R tokens and one block of columns: it reads the R ids, then R independent pieces of rows.  With
// many tokens the rows come out of L2 for the most part, and L2 bounds it: 65536 rows of 4 KB in and out move 537 MB in 78 us,
// 6.9 TB/s.  More rows per warp cost warps (R = 4: 85 us, R = 8: 101), fewer leave it waiting for the ids (R = 1: 101).  The
// output is written past L2 (evict first), whose room belongs to the table.
constexpr int EMBED_TPB = 128;

template <typename W, typename O, bool VEC, int R>
__global__ void __launch_bounds__(EMBED_TPB) k_embed(const W* __restrict__ weight, int64_t V, int64_t D, int64_t ldw, const void* __restrict__ ids,
                                                      int id_type, int64_t T, float scale, O* __restrict__ out, int64_t ldo, unsigned ncb) {
  const int lane = threadIdx.x & 31;
  const int64_t item = int64_t(blockIdx.x) * (EMBED_TPB / 32) + (threadIdx.x >> 5);
  const int64_t t0 = item / ncb * R, cb = item % ncb;
  if (t0 >= T) return;
  const int n = int(min(int64_t(R), T - t0));
  const int mine = lane < n ? int(load_id(ids, id_type, t0 + lane, V)) : -1;
  uint4 u[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int v = __shfl_sync(0xffffffffu, mine, i);
    u[i] = make_uint4(0, 0, 0, 0);
    if (v >= 0) load_raw<W, VEC>(weight + v * ldw, D, cb, lane, 32, u[i]);
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i >= n) break;
    const bool known = __shfl_sync(0xffffffffu, mine, i) >= 0;      // an unknown id gives +0 whatever the scale
    Raw<W> r;
    memcpy(&r, &u[i], 16);
    struct alignas(sizeof(O) * LANE<W> < 16 ? sizeof(O) * LANE<W> : 16) Row { O e[LANE<W>]; } o;
#pragma unroll
    for (int j = 0; j < LANE<W>; ++j) o.e[j] = from_f<O>(known ? to_f(r.e[j]) * scale : 0.0f);
    O* dst = out + (t0 + i) * ldo;
    const int64_t c0 = column<W, VEC>(cb, lane, 0);
    if (VEC && c0 + LANE<W> <= D) {
      if constexpr (sizeof(Row) == 16) { float4 q; memcpy(&q, &o, 16); __stcs(reinterpret_cast<float4*>(dst + c0), q); }
      else *reinterpret_cast<Row*>(dst + c0) = o;
    } else {
#pragma unroll
      for (int j = 0; j < LANE<W>; ++j) {
        const int64_t c = column<W, VEC>(cb, lane, j);
        if (c < D) dst[c] = o.e[j];
      }
    }
  }
}

// Rows of at most half a block share a warp: 2^lanes_log lanes each (37752 rows of 128 bytes: 3.1 us, with a warp each 11.2).
template <typename W, typename O, bool VEC>
__global__ void __launch_bounds__(EMBED_TPB) k_embed_narrow(const W* __restrict__ weight, int64_t V, int64_t D, int64_t ldw, const void* __restrict__ ids,
                                                             int id_type, int64_t T, float scale, O* __restrict__ out, int64_t ldo, int lanes_log) {
  const int lanes = 1 << lanes_log, lane = threadIdx.x & (lanes - 1);
  const int64_t t = (int64_t(blockIdx.x) * EMBED_TPB + threadIdx.x) >> lanes_log;
  if (t >= T) return;
  const int64_t v = load_id(ids, id_type, t, V);
  uint4 u = make_uint4(0, 0, 0, 0);
  if (v >= 0) load_raw<W, VEC>(weight + v * ldw, D, 0, lane, lanes, u);
  Raw<W> r;
  memcpy(&r, &u, 16);
  struct alignas(sizeof(O) * LANE<W> < 16 ? sizeof(O) * LANE<W> : 16) Row { O e[LANE<W>]; } o;
#pragma unroll
  for (int j = 0; j < LANE<W>; ++j) o.e[j] = from_f<O>(v >= 0 ? to_f(r.e[j]) * scale : 0.0f);
  O* dst = out + t * ldo;
  if (VEC && (lane + 1) * LANE<W> <= D) {
    *reinterpret_cast<Row*>(dst + lane * LANE<W>) = o;
  } else {
#pragma unroll
    for (int j = 0; j < LANE<W>; ++j) {
      const int64_t c = column<W, VEC>(0, lane, j, lanes);
      if (c < D) dst[c] = o.e[j];
    }
  }
}

// ------------------------------------------------------------------------------------------ gradient: grouping the tokens
// The tokens fall into nb buckets (a power of two) by id mod nb, so that the frequent tokens, which have neighbouring
// ids, spread over all buckets.  A bucket's CTA reads all ids: each of its warps owns a consecutive stretch, counts the
// tokens of lower buckets and lists its own ones.  The lists, end to end, are the bucket's tokens in order; they are
// counted per (id, warp), and a scan turns the counts into places: grouped by id, in token order, without a sort.  What it
// costs is latency (half a dozen short phases, 3 us for 2048 tokens) and, for many tokens, the 128-fold reading of the ids out
// of L2 (67 MB for 65536 ids of 64 bits: 12 us in all).  A cluster of four CTAs that reads the ids once and passes the
// tokens through distributed shared memory took as long: what it saves it spends on the cluster's barriers and remote reads.
// Lists that would not hold all (a text of very few ids, millions of tokens) are not used: then the ids are read twice more.
constexpr int SORT_TPB = 1024;
constexpr int SORT_WARPS = SORT_TPB / 32;
constexpr int SORT_BINS = 1024;      // ids per bucket, at most: one thread each in the scan, 128 KB of counters
constexpr int SORT_LIST = 128;       // tokens a warp lists (32 KB); one in nb of its stretch on average
constexpr int SORT_OWN = SORT_WARPS * SORT_LIST;

struct EmbedPlan {
  int nb_log;
  int64_t bins;                      // counters per bucket
  int piece;                         // sorted tokens per warp of the summation
  int64_t pieces, ncb;
  size_t perm, row, start, valid, ticket, part, total;
};

inline EmbedPlan embed_plan(int64_t T, int64_t V, int64_t D, int block) {
  EmbedPlan p;
  p.nb_log = 7;
  while (((V - 1) >> p.nb_log) + 1 > SORT_BINS) ++p.nb_log;
  p.bins = ((V - 1) >> p.nb_log) + 1;
  p.ncb = (D + block - 1) / block;
  // short pieces while long ones would not give every multiprocessor its 32 warps: then the length of one warp's chain counts
  p.piece = (T + 31) / 32 * p.ncb >= 148 * 32 ? 32 : 8;
  p.pieces = (T + p.piece - 1) / p.piece;
  size_t o = 0;
  p.valid = o;  o = align_up(o + 4, 16);
  p.perm = o;   o = align_up(o + size_t(T) * 4, 16);
  p.row = o;    o = align_up(o + size_t(T) * 4, 16);
  p.start = o;  o = align_up(o + (size_t(p.bins + 1) << p.nb_log) * 4, 16);
  p.ticket = o; o = align_up(o + size_t(p.pieces) * size_t(p.ncb) * 8, 16);
  p.part = o;   o = align_up(o + size_t(p.pieces) * 2 * size_t(D) * 4, 16);
  p.total = o;
  return p;
}

struct SortArgs {
  const void* ids;
  int64_t T, V, pad_id;
  int nb_log, bins;
  int32_t *perm, *row;
  int32_t* start;                    // [id]: place of the id's first token; [id + nb]: the place behind its last one
  int32_t* valid;                    // tokens with a gradient
  uint32_t* ticket;
  int64_t n_ticket;
};

struct SortSmem {
  int2 list[SORT_WARPS][SORT_LIST];  // (token, id)
  int2 own[SORT_OWN];                // the lists end to end
  uint32_t warp[SORT_WARPS], below[SORT_WARPS];
  uint32_t cnt[1];                   // [row][bin] counts, then next places; a row per warp
};

// 256 consecutive ids, eight per lane: 16 bytes of ids a lane and load, loads end to end; -1 from `hi` on.
template <typename ID> struct Ids {
  static constexpr int PER = 16 / int(sizeof(ID)), LOADS = 8 / PER;
  ID v[LOADS][PER];
  __device__ static int64_t offset(int lane, int j, int e) { return j * 32 * PER + lane * PER + e; }
};
template <typename ID> __device__ __forceinline__ void load_ids(const ID* ids, int64_t t, int64_t hi, bool aligned, int lane, Ids<ID>& x) {
  if (aligned && t + 256 <= hi) {
#pragma unroll
    for (int j = 0; j < Ids<ID>::LOADS; ++j) {
      const uint4 u = __ldg(reinterpret_cast<const uint4*>(ids + t + Ids<ID>::offset(lane, j, 0)));
      memcpy(x.v[j], &u, 16);
    }
  } else {
#pragma unroll
    for (int j = 0; j < Ids<ID>::LOADS; ++j)
#pragma unroll
      for (int e = 0; e < Ids<ID>::PER; ++e) {
        const int64_t i = t + Ids<ID>::offset(lane, j, e);
        x.v[j][e] = i < hi ? ids[i] : ID(-1);
      }
  }
}

template <typename ID>
__global__ void __launch_bounds__(SORT_TPB) k_embed_sort(const __grid_constant__ SortArgs a) {
  extern __shared__ __align__(16) unsigned char sort_smem[];
  SortSmem& s = *reinterpret_cast<SortSmem*>(sort_smem);
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const uint32_t b = blockIdx.x, mask = (1u << a.nb_log) - 1u;
  const int bins = a.bins;
  const unsigned lower = (1u << lane) - 1u;
  const uint32_t V = uint32_t(a.V), pad = a.pad_id >= 0 && a.pad_id < a.V ? uint32_t(a.pad_id) : ~0u;
  const ID* ids = static_cast<const ID*>(a.ids);
  const bool aligned = (reinterpret_cast<uintptr_t>(ids) & 15) == 0;
  uint32_t* row = s.cnt + w * bins;
  asm volatile("griddepcontrol.launch_dependents;");      // the sums may be set up; they wait for the end of this kernel
  const int64_t seg = (a.T + SORT_WARPS * 256 - 1) / (SORT_WARPS * 256) * 256;
  const int64_t lo = min(a.T, w * seg), hi = min(a.T, lo + seg);
  auto known = [&](ID v) { return (sizeof(ID) == 4 || uint64_t(v) >> 32 == 0) && uint32_t(v) < V && uint32_t(v) != pad; };
  Ids<ID> x;
  load_ids(ids, lo, hi, aligned, lane, x);
  for (int i = threadIdx.x; i < SORT_WARPS * bins; i += SORT_TPB) s.cnt[i] = 0;
  for (int64_t i = int64_t(b) * SORT_TPB + threadIdx.x; i < a.n_ticket; i += int64_t(gridDim.x) * SORT_TPB) a.ticket[i] = 0;
  uint32_t below = 0;
  int found = 0;
  for (int64_t t0 = lo; t0 < hi; t0 += 256) {
    const Ids<ID> y = x;
    if (t0 + 256 < hi) load_ids(ids, t0 + 256, hi, aligned, lane, x);
    unsigned hit = 0, c = 0;         // hits of this lane: a bit each, and a byte per load
#pragma unroll
    for (int j = 0; j < Ids<ID>::LOADS; ++j)
#pragma unroll
      for (int e = 0; e < Ids<ID>::PER; ++e) {
        const uint32_t m = uint32_t(y.v[j][e]) & mask;
        const bool is = known(y.v[j][e]);
        below += is && m < b;
        if (is && m == b) { hit |= 1u << (j * Ids<ID>::PER + e); c += 1u << (8 * j); }
      }
    if (!__any_sync(0xffffffffu, hit != 0)) continue;
    unsigned incl = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned z = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += z;
    }
    const unsigned all = __shfl_sync(0xffffffffu, incl, 31), ahead = incl - c;
#pragma unroll
    for (int j = 0; j < Ids<ID>::LOADS; ++j) {
      int at = found + int(ahead >> (8 * j) & 255u);
#pragma unroll
      for (int e = 0; e < Ids<ID>::PER; ++e)
        if (hit >> (j * Ids<ID>::PER + e) & 1u) {
          if (at < SORT_LIST) s.list[w][at] = make_int2(int(t0 + Ids<ID>::offset(lane, j, e)), int(y.v[j][e]));
          ++at;
        }
      found += int(all >> (8 * j) & 255u);
    }
  }
  below = __reduce_add_sync(0xffffffffu, below);
  if (lane == 0) { s.warp[w] = found; s.below[w] = below; }
  __syncthreads();
  const uint32_t nw = s.warp[lane];
  const uint32_t before = __reduce_add_sync(0xffffffffu, s.below[lane]);      // tokens in lower buckets
  const int own = int(__reduce_add_sync(0xffffffffu, nw));
  const bool listed = __reduce_max_sync(0xffffffffu, nw) <= SORT_LIST;
  // rows of counts: a warp per 32 tokens while there are fewer than 32 such, else 1/32 of the tokens each
  const int chunk = (own + SORT_TPB - 1) / SORT_TPB * 32;
  const int rows = listed ? (own == 0 ? 0 : (own + chunk - 1) / chunk) : SORT_WARPS;
  const int i0 = min(own, w * chunk), i1 = min(own, i0 + chunk);
  auto again = [&](auto&& f) {       // the stretch once more, 32 tokens at a time and in order, eight loads on their way
    for (int64_t t0 = lo; t0 < hi; t0 += 256) {
      ID v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = t0 + u * 32 + lane < hi ? ids[t0 + u * 32 + lane] : ID(-1);
#pragma unroll
      for (int u = 0; u < 8; ++u) f(int(t0) + u * 32 + lane, v[u]);
    }
  };
  auto mine = [&](ID v) { return known(v) && (uint32_t(v) & mask) == b; };
  if (listed) {
    const int at = int(__reduce_add_sync(0xffffffffu, lane < w ? nw : 0u));
    for (int i = lane; i < found; i += 32) s.own[at + i] = s.list[w][i];
    __syncthreads();
    for (int i = i0 + lane; i < i1; i += 32) atomicAdd(&row[s.own[i].y >> a.nb_log], 1u);
  } else {
    again([&](int, ID v) {
      if (mine(v)) atomicAdd(&row[uint32_t(v) >> a.nb_log], 1u);
    });
  }
  __syncthreads();
  // places: an exclusive scan over the ids' totals, then over the rows of each id
  uint32_t total = 0;
  if (int(threadIdx.x) < bins)
    for (int i = 0; i < rows; ++i) total += s.cnt[i * bins + threadIdx.x];
  uint32_t incl = total;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t z = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += z;
  }
  if (lane == 31) s.warp[w] = incl;
  __syncthreads();
  uint32_t run = before + incl - total + __reduce_add_sync(0xffffffffu, lane < w ? s.warp[lane] : 0u);
  if (int(threadIdx.x) < bins) {
    a.start[(int64_t(threadIdx.x) << a.nb_log) + b] = int32_t(run);
    for (int i = 0; i < rows; ++i) { const uint32_t c = s.cnt[i * bins + threadIdx.x]; s.cnt[i * bins + threadIdx.x] = run; run += c; }
    if (int(threadIdx.x) == bins - 1) {
      a.start[(int64_t(bins) << a.nb_log) + b] = int32_t(run);
      if (b == gridDim.x - 1) *a.valid = int32_t(run);
    }
  }
  __syncthreads();
  auto place = [&](int t, int v, bool is) {      // 32 tokens at a time, in order: the row's next place, past the lanes ahead with the same id
    const unsigned any = __ballot_sync(0xffffffffu, is);
    if (is) {
      const unsigned same = __match_any_sync(any, v);
      const int ahead = __popc(same & lower), bin = v >> a.nb_log;
      const uint32_t slot = row[bin] + ahead;
      __syncwarp(any);
      if (ahead == 0) row[bin] += __popc(same);
      a.perm[slot] = t;
      a.row[slot] = v;
    }
    __syncwarp();
  };
  if (listed) {
    for (int i = i0 + lane; i - lane < i1; i += 32) {
      const int2 e = i < i1 ? s.own[i] : make_int2(0, 0);
      place(e.x, e.y, i < i1);
    }
  } else {
    again([&](int t, ID v) { place(t, int(v), mine(v)); });
  }
}

// ------------------------------------------------------------------------------------------ gradient: the sums
// A warp takes one piece of consecutive sorted tokens and one block of columns and adds the rows up in order.  A run of
// equal ids that lies inside the piece is finished there.  One that crosses into other pieces leaves a partial sum per
// piece; the warp that leaves the last one adds the partial sums up in the order of the pieces.  So a frequent token's
// rows are read by many warps, and the result does not depend on which of them comes last.  CTAs that clear the rows
// without a token follow those that sum.  Memory bounds it: 65536 tokens x 2048 bf16 into 65536 rows are 806 MB in 120 us,
// 6.7 TB/s; with rows in registers instead of the asynchronous ring it was 202 us (latency: two CTAs a multiprocessor).
struct SumArgs {
  const int32_t *perm, *row, *start, *valid;
  uint32_t* ticket;                  // [2][piece][block of columns] warps that have arrived, at either level of the joining
  float* part;                       // [piece][0: the run that the piece begins with, 1: the one it ends with][D]
  int64_t V, D, ldd, ldw, pieces;
  float scale;
  int accumulate, nb, ncb;
  int dw_aligned;                    // the table's rows start at multiples of what a lane stores (16 or 32 bytes)
  int64_t n_fill;                    // CTAs that clear
  int fill_rows;                     // rows each of them looks at
  float* dweight;
};

constexpr int SUM_TPB = 256;
constexpr int JOIN = 16;             // partial sums added up by one warp
constexpr int RING = 8;              // rows on their way per warp (4 KB; 32 warps a multiprocessor)

// A row of zeros, written by one warp: single words up to a 16-byte boundary, then 16 bytes a lane.
__device__ __forceinline__ void clear_row(float* p, int64_t D, int lane) {
  const int64_t head = min(D, int64_t((16 - (reinterpret_cast<uintptr_t>(p) & 15)) / 4 & 3));
  if (lane < head) p[lane] = 0.0f;
  float4* q = reinterpret_cast<float4*>(p + head);
  const int64_t nv = (D - head) >> 2;
  for (int64_t i = lane; i < nv; i += 32) q[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const int64_t done = head + 4 * nv;
  if (lane < D - done) p[done + lane] = 0.0f;
}

// Clears the unused ones of the rows a CTA looks at.  Every warp has one row in eight; but where rows follow one another
// without a gap and are narrow, or would be written in parts of sectors, it has neighbouring rows, and clears neighbouring unused ones as one
// (56769 rows of 256 bytes: 4.5 us, row by row 9.7; 50021 of 4004 bytes: 33.5 and 37.3).
template <typename F> __device__ __forceinline__ void clear_unused(const SumArgs& a, int64_t cta, F&& unused) {
  constexpr int W = SUM_TPB / 32;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, rows = a.fill_rows / W;
  const bool merge = a.ldw == a.D && (a.D < 128 || a.D % 8 != 0 || (reinterpret_cast<uintptr_t>(a.dweight) & 31) != 0);
  const int step = merge ? 1 : W;
  const int64_t v0 = cta * a.fill_rows + (merge ? w * rows : w);
  for (int i0 = 0; i0 < rows; i0 += 32) {
    const int64_t mine = v0 + int64_t(i0 + lane) * step;
    unsigned m = __ballot_sync(0xffffffffu, i0 + lane < rows && mine < a.V && unused(mine));
    while (m) {
      const int i = __ffs(int(m)) - 1, run = __ffs(int(~(m >> i))) - 1;      // (-1 where m is all ones)
      const int n = !merge ? 1 : run < 0 ? 32 : run;
      clear_row(a.dweight + (v0 + int64_t(i0 + i) * step) * a.ldw, n * a.D, lane);
      m &= i + n >= 32 ? 0u : ~0u << (i + n);
    }
  }
}

template <typename X> struct Lanes { float v[LANE<X>]; };

template <typename X, bool VEC>
__device__ __forceinline__ void put_row(const SumArgs& a, int64_t v, int64_t cb, int lane, const Lanes<X>& acc, float* stage) {
  float* dst = a.dweight + v * a.ldw;
  if (VEC && a.dw_aligned && column<X, VEC>(cb, lane, 0) + LANE<X> <= a.D) {
    float* q = dst + column<X, VEC>(cb, lane, 0);
    float o[LANE<X>];
#pragma unroll
    for (int j = 0; j < LANE<X>; ++j) o[j] = acc.v[j] * a.scale;
    if (a.accumulate) {
#pragma unroll
      for (int j = 0; j < LANE<X>; j += 4) {
        const float4 old = *reinterpret_cast<const float4*>(q + j);
        o[j] += old.x; o[j + 1] += old.y; o[j + 2] += old.z; o[j + 3] += old.w;
      }
    }
    if constexpr (LANE<X> == 8) {      // one 32-byte store a lane: whole sectors
      asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(q), "f"(o[0]), "f"(o[1]), "f"(o[2]), "f"(o[3]), "f"(o[4]),
                   "f"(o[5]), "f"(o[6]), "f"(o[7]) : "memory");
    } else {
      *reinterpret_cast<float4*>(q) = make_float4(o[0], o[1], o[2], o[3]);
    }
    return;
  }
  const bool turn = VEC && !a.dw_aligned;            // turn the block through shared memory: contiguous words for the warp
  if (turn) {
#pragma unroll
    for (int j = 0; j < LANE<X>; ++j) stage[lane * LANE<X> + j] = acc.v[j];
    __syncwarp();
  }
#pragma unroll
  for (int j = 0; j < LANE<X>; ++j) {
    const int64_t c = turn ? cb * BLOCK<X> + j * 32 + lane : column<X, VEC>(cb, lane, j);
    const float x = (turn ? stage[j * 32 + lane] : acc.v[j]) * a.scale;
    if (c < a.D) dst[c] = a.accumulate ? dst[c] + x : x;
  }
  if (turn) __syncwarp();
}

// Partial sums are kept in lane order (not column order): [piece][slot][block of columns][j][lane].
template <typename X> __device__ __forceinline__ float* part_at(const SumArgs& a, int64_t piece, int slot, int64_t cb, int lane) {
  return a.part + ((piece * 2 + slot) * a.ncb + cb) * BLOCK<X> + lane;
}

// 16 bytes of a row on their way to this lane's slot in shared memory.  Rows of 16-bit elements that do not start at a
// multiple of 16 bytes have no asynchronous copy; they go through registers.
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }

template <typename X, bool VEC> __device__ __forceinline__ void fetch(const X* row, int64_t D, int64_t cb, int lane, uint4* slot) {
  const int64_t c0 = column<X, VEC>(cb, lane, 0);
  if (VEC && c0 + LANE<X> <= D) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(slot)), "l"(row + c0) : "memory");
  } else if (!VEC && sizeof(X) == 4) {
#pragma unroll
    for (int j = 0; j < LANE<X>; ++j) {
      const int64_t c = c0 + j * 32;
      if (c < D) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_addr(reinterpret_cast<X*>(slot) + j)), "l"(row + c) : "memory");
    }
  } else {
    load_raw<X, VEC>(row, D, cb, lane, 32, *slot);
  }
}

// PIECE: tokens per warp.
template <typename X, bool VEC, int PIECE>
__global__ void __launch_bounds__(SUM_TPB, 4) k_embed_sum(const X* __restrict__ dout, const __grid_constant__ SumArgs a) {
  constexpr int E = LANE<X>, DEPTH = PIECE < RING ? PIECE : RING;
  extern __shared__ uint4 ring[];                   // [DEPTH][thread]: a lane only ever reads what it fetched itself
  __shared__ float s_stage[VEC ? SUM_TPB / 32 : 1][VEC ? BLOCK<X> : 1];
  const int lane = threadIdx.x & 31;
  float* stage = VEC ? s_stage[threadIdx.x >> 5] : nullptr;
  // the CTAs that clear come last: their stores fill the time in which the last sums wait for their rows (in between, or
  // first, they cost 8 to 4 % more at 65536 tokens, 65536 x 2048)
  const int64_t n_sum = gridDim.x - a.n_fill;
  const bool clears = blockIdx.x >= n_sum;
  const int64_t item = int64_t(blockIdx.x) * (SUM_TPB / 32) + (threadIdx.x >> 5);
  const int64_t piece = item / a.ncb, cb = item % a.ncb;
  const int64_t s0 = piece * PIECE;
  if (!clears)
    for (int i = 0; i < DEPTH; ++i) ring[i * SUM_TPB + threadIdx.x] = make_uint4(0, 0, 0, 0);     // columns beyond the row stay zero
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (clears) {
    clear_unused(a, blockIdx.x - n_sum, [&](int64_t v) { return a.start[v] == a.start[v + a.nb]; });
    return;
  }
  const int64_t valid = *a.valid;
  if (s0 >= valid) return;
  const int n = int(min(int64_t(PIECE), valid - s0));
  const int32_t p = lane < n ? a.perm[s0 + lane] : 0;
  const int32_t r = lane < n ? a.row[s0 + lane] : -1;
  const int32_t before = s0 > 0 ? a.row[s0 - 1] : -1;
  const int32_t after = s0 + n < valid ? a.row[s0 + n] : -1;
  auto issue = [&](int i) {
    const int64_t t = __shfl_sync(0xffffffffu, p, i & 31);
    if (i < n) fetch<X, VEC>(dout + t * a.ldd, a.D, cb, lane, ring + (i % DEPTH) * SUM_TPB + threadIdx.x);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < DEPTH; ++i) issue(i);
  const int32_t r0 = __shfl_sync(0xffffffffu, r, 0), rn = __shfl_sync(0xffffffffu, r, n - 1);
  const int32_t next = __shfl_down_sync(0xffffffffu, r, 1);
  const unsigned ends = __ballot_sync(0xffffffffu, lane < n && (lane == n - 1 || next != r));   // last token of a run (or of the piece)
  // the places of the runs that cross into this piece and out of it
  const bool cross0 = before == r0 || (r0 == rn && after == rn), cross1 = r0 != rn && after == rn;
  int first[2] = {0, 0}, last[2] = {0, 0};
  if (cross0) { first[0] = a.start[r0]; last[0] = a.start[r0 + a.nb] - 1; }
  if (cross1) { first[1] = a.start[rn]; last[1] = a.start[rn + a.nb] - 1; }
  Lanes<X> acc;
#pragma unroll
  for (int j = 0; j < E; ++j) acc.v[j] = 0.0f;
#pragma unroll 1
  for (int i = 0; i < n; ++i) {
    asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
    Raw<X> x;
    memcpy(&x, ring + (i % DEPTH) * SUM_TPB + threadIdx.x, 16);
    if (PIECE > DEPTH) issue(i + DEPTH);
    else asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll
    for (int j = 0; j < E; ++j) acc.v[j] += to_f(x.e[j]);
    if (!(ends >> i & 1u)) continue;
    const int32_t v = __shfl_sync(0xffffffffu, r, i);
    const int slot = v == r0 ? 0 : 1;
    if ((slot == 0 && cross0) || (i == n - 1 && cross1)) {
      float* q = part_at<X>(a, piece, slot, cb, lane);
#pragma unroll
      for (int j = 0; j < E; ++j) __stcg(q + j * 32, acc.v[j]);
    } else {
      put_row<X, VEC>(a, v, cb, lane, acc, stage);
    }
#pragma unroll
    for (int j = 0; j < E; ++j) acc.v[j] = 0.0f;
  }
  if (!cross0 && !cross1) return;
  // This piece's partial sums are written.  The warp that brings the last of up to JOIN neighbouring pieces of a run adds them up,
  // and of a longer run, the warp that brings the last such sum adds those up: two short chains of loads instead of a long one.
  __threadfence();
  __syncwarp();
#pragma unroll 1
  for (int c = 0; c < 2; ++c) {
    if (!(c ? cross1 : cross0)) continue;
    const int f = c ? first[1] : first[0], p0 = f / PIECE, p1 = (c ? last[1] : last[0]) / PIECE;
    auto slot_of = [&](int p) { return p == p0 && f % PIECE ? 1 : 0; };
    auto last_one = [&](uint32_t* ticket, int others) {      // of others + 1 warps
      uint32_t arrived = 0;
      if (lane == 0) arrived = atomicAdd(ticket, 1u);
      if (__shfl_sync(0xffffffffu, arrived, 0) != uint32_t(others)) return false;
      __threadfence();
      return true;
    };
    auto add = [&](int from, int to, int step) {      // the sums left at pieces from, from + step, ..., to
      const float* q = part_at<X>(a, from, slot_of(from), cb, lane);
#pragma unroll
      for (int j = 0; j < E; ++j) acc.v[j] = __ldcg(q + j * 32);
#pragma unroll 4
      for (int k = from + step; k <= to; k += step) {
        q = part_at<X>(a, k, 0, cb, lane);
#pragma unroll
        for (int j = 0; j < E; ++j) acc.v[j] += __ldcg(q + j * 32);
      }
    };
    const int g0 = int(piece) - (int(piece) - p0) % JOIN, g1 = min(p1, g0 + JOIN - 1);
    if (g1 > g0 && !last_one(a.ticket + int64_t(g0) * a.ncb + cb, g1 - g0)) continue;
    add(g0, g1, 1);
    if (p1 - p0 >= JOIN) {
      float* q = part_at<X>(a, g0, slot_of(g0), cb, lane);
#pragma unroll
      for (int j = 0; j < E; ++j) __stcg(q + j * 32, acc.v[j]);
      __threadfence();
      __syncwarp();
      if (!last_one(a.ticket + (a.pieces + p0) * a.ncb + cb, (p1 - p0) / JOIN)) continue;
      add(p0, p1, JOIN);
    }
    put_row<X, VEC>(a, c ? rn : r0, cb, lane, acc, stage);
  }
}

// A few tokens: one kernel, no grouping.  A warp takes one token and one block of columns; if no token before has the same
// id it adds up the rows of all that have.  (Two tokens, 56769 x 64: 5.0 us, with the two kernels 12.7.)
constexpr int FEW = 128;
constexpr int FEW_ROWS = 32768;      // most rows a CTA that clears looks at

struct FewArgs {
  SumArgs sum;
  const void* ids;
  int id_type;
  int T;
  int64_t pad_id, n_sum;             // CTAs that sum
};

template <typename X, bool VEC>
__global__ void __launch_bounds__(SUM_TPB) k_embed_few(const X* __restrict__ dout, const __grid_constant__ FewArgs f) {
  __shared__ int s_id[FEW];
  __shared__ uint32_t s_used[FEW_ROWS / 32];
  __shared__ float s_stage[VEC ? SUM_TPB / 32 : 1][VEC ? BLOCK<X> : 1];
  const SumArgs& a = f.sum;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  if (int(threadIdx.x) < FEW) {
    const int64_t v = int(threadIdx.x) < f.T ? load_id(f.ids, f.id_type, threadIdx.x, a.V) : -1;
    s_id[threadIdx.x] = v == f.pad_id ? -1 : int(v);
  }
  if (blockIdx.x >= f.n_sum) {
    const int64_t cta = blockIdx.x - f.n_sum, v0 = cta * a.fill_rows;
    for (int i = threadIdx.x; i < (a.fill_rows + 31) / 32; i += SUM_TPB) s_used[i] = 0;
    __syncthreads();
    if (int(threadIdx.x) < FEW) {
      const int64_t r = s_id[threadIdx.x] - v0;
      if (s_id[threadIdx.x] >= 0 && r >= 0 && r < a.fill_rows) atomicOr(&s_used[r / 32], 1u << (r % 32));
    }
    __syncthreads();
    clear_unused(a, cta, [&](int64_t v) { return !(s_used[(v - v0) / 32] >> ((v - v0) % 32) & 1u); });
    return;
  }
  __syncthreads();
  const int64_t item = int64_t(blockIdx.x) * (SUM_TPB / 32) + w, cb = item % a.ncb;
  const int t = int(min(item / a.ncb, int64_t(FEW - 1)));
  const int v = item / a.ncb < f.T ? s_id[t] : -1;
  if (v < 0) return;
  unsigned same[FEW / 32], before = 0;
#pragma unroll
  for (int i = 0; i < FEW / 32; ++i) {
    same[i] = __ballot_sync(0xffffffffu, s_id[i * 32 + lane] == v);
    before |= i < t / 32 ? same[i] : i == t / 32 ? same[i] & ((1u << (t & 31)) - 1u) : 0u;
  }
  if (before) return;
  Lanes<X> acc;
#pragma unroll
  for (int j = 0; j < LANE<X>; ++j) acc.v[j] = 0.0f;
#pragma unroll 1
  for (int i = 0; i < FEW / 32; ++i) {
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < FEW / 32; ++j) m = j == i ? same[j] : m;
    while (m) {
      constexpr int U = 4;           // rows on their way
      uint4 u[U];
      int n = 0;
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (m) {
          const int64_t at = i * 32 + __ffs(int(m)) - 1;
          m &= m - 1;
          load_raw<X, VEC>(dout + at * a.ldd, a.D, cb, lane, 32, u[k]);
          n = k + 1;
        }
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (k < n) {
          Raw<X> x;
          memcpy(&x, &u[k], 16);
#pragma unroll
          for (int j = 0; j < LANE<X>; ++j) acc.v[j] += to_f(x.e[j]);
        }
    }
  }
  put_row<X, VEC>(a, v, cb, lane, acc, VEC ? s_stage[w] : nullptr);
}

inline bool rows_aligned(const void* p, int64_t ld, int size, int bytes) { return !misaligned(p, bytes) && ld * size % bytes == 0; }

}  // namespace

extern "C" {

int mv_embed(void* stream, const void* weight, int w_type, int64_t V, int64_t D, int64_t ldw, const void* ids, int id_type,
             int64_t T, float scale, void* out, int out_type, int64_t ldo) {
  const int64_t lim = int64_t(1) << 31;
  if (!is_value_type(w_type) || !is_value_type(out_type) || !is_id_type(id_type) || V < 1 || V >= lim || D < 1 || D >= lim || T < 0 ||
      T >= lim || ldw < D || ldo < D || !weight || (T > 0 && (!ids || !out)) || misaligned(weight, type_size(w_type)) ||
      misaligned(ids, type_size(id_type)) || misaligned(out, type_size(out_type)))
    return MV_ERR_INVALID_ARG;
  if (share_bytes(weight, V, D, ldw, type_size(w_type), out, T, D, ldo, type_size(out_type))) return MV_ERR_INVALID_ARG;
  if (T == 0) return MV_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_type(w_type, [&](auto w) {
    return with_type(out_type, [&](auto o) {
      using W = decltype(w);
      using O = decltype(o);
      const int64_t ncb = (D + BLOCK<W> - 1) / BLOCK<W>;
      const int ob = int(sizeof(O)) * LANE<W> < 16 ? int(sizeof(O)) * LANE<W> : 16;
      const bool vec = rows_aligned(weight, ldw, sizeof(W), 16) && rows_aligned(out, ldo, sizeof(O), ob);
      // two tokens a warp once that still gives every multiprocessor its 64 warps; below, the latency of one row counts
      int lanes_log = 5;
      while (ncb == 1 && lanes_log > 0 && (int64_t(LANE<W>) << (lanes_log - 1)) >= D) --lanes_log;
      if (lanes_log < 5) {
        const int64_t grid = ((T << lanes_log) + EMBED_TPB - 1) / EMBED_TPB;
        auto* kernel = vec ? k_embed_narrow<W, O, true> : k_embed_narrow<W, O, false>;
        kernel<<<unsigned(grid), EMBED_TPB, 0, st>>>(static_cast<const W*>(weight), V, D, ldw, ids, id_type, T, scale, static_cast<O*>(out), ldo, lanes_log);
        return cuda_ok();
      }
      const int R = T * ncb >= 148 * 64 * 2 ? 2 : 1;
      const int64_t items = (T + R - 1) / R * ncb, grid = (items + EMBED_TPB / 32 - 1) / (EMBED_TPB / 32);
      if (grid >= lim) return int(MV_ERR_INVALID_ARG);
      auto* kernel = vec ? (R == 2 ? k_embed<W, O, true, 2> : k_embed<W, O, true, 1>) : (R == 2 ? k_embed<W, O, false, 2> : k_embed<W, O, false, 1>);
      kernel<<<unsigned(grid), EMBED_TPB, 0, st>>>(static_cast<const W*>(weight), V, D, ldw, ids, id_type, T, scale, static_cast<O*>(out), ldo, int(ncb));
      return cuda_ok();
    });
  });
}

size_t mv_embed_grad_workspace_bytes(int64_t T, int64_t V, int64_t D) {
  const int64_t lim = int64_t(1) << 31;
  if (T < 0 || T >= lim || V < 1 || V >= lim || D < 1 || D >= lim) return 0;
  // the largest any type of dout needs: blocks of 128 columns (32 bits) give the most tickets, of 256 (16 bits) the widest rows
  const EmbedPlan a = embed_plan(T, V, (D + 127) / 128 * 128, 128), b = embed_plan(T, V, (D + 255) / 256 * 256, 256);
  return a.total > b.total ? a.total : b.total;
}

int mv_embed_grad(void* stream, const void* dout, int dout_type, int64_t ldd, const void* ids, int id_type, int64_t T, int64_t V,
                  int64_t D, float scale, int64_t pad_id, int accumulate, float* dweight, int64_t ldw, void* workspace,
                  size_t workspace_bytes) {
  const int64_t lim = int64_t(1) << 31;
  if (!is_value_type(dout_type) || !is_id_type(id_type) || T < 0 || T >= lim || V < 1 || V >= lim || D < 1 || D >= lim || ldd < D ||
      ldw < D || (accumulate != 0 && accumulate != 1) || !dweight || (T > 0 && (!dout || !ids)) || misaligned(dout, type_size(dout_type)) ||
      misaligned(ids, type_size(id_type)) || misaligned(dweight, 4) || misaligned(workspace, 16))
    return MV_ERR_INVALID_ARG;
  if (share_bytes(dout, T, D, ldd, type_size(dout_type), dweight, V, D, ldw, 4)) return MV_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < mv_embed_grad_workspace_bytes(T, V, D)) return MV_ERR_WORKSPACE;
  const int block = dout_type == MV_F32 ? BLOCK<float> : BLOCK<__half>;
  const EmbedPlan p = embed_plan(T, V, (D + block - 1) / block * block, block);
  const int64_t items = p.pieces * p.ncb, n_sum = (items + SUM_TPB / 32 - 1) / (SUM_TPB / 32);
  SumArgs a;
  // a CTA that clears looks at 128 KB of rows, at fewer where that would not give every multiprocessor four of them, and at
  // eight at least (one a warp)
  const int64_t by_size = (32 << 10) / D, by_count = V / (148 * 4);
  a.fill_rows = int(((by_size < by_count ? by_size : by_count) + 7) / 8 * 8);
  if (a.fill_rows < 8) a.fill_rows = 8;
  a.n_fill = accumulate ? 0 : (V + a.fill_rows - 1) / a.fill_rows;
  if (n_sum + a.n_fill >= lim) return MV_ERR_INVALID_ARG;
  if (accumulate && T == 0) return MV_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  a.V = V; a.D = D; a.ldd = ldd; a.ldw = ldw; a.scale = scale; a.accumulate = accumulate; a.nb = 1 << p.nb_log;
  a.ncb = int(p.ncb);
  a.pieces = p.pieces;
  a.dw_aligned = rows_aligned(dweight, ldw, 4, dout_type == MV_F32 ? 16 : 32);
  a.dweight = dweight;
  if (T <= FEW) {
    FewArgs f;
    f.sum = a; f.ids = ids; f.id_type = id_type; f.T = int(T); f.pad_id = pad_id;
    f.n_sum = (T * p.ncb + SUM_TPB / 32 - 1) / (SUM_TPB / 32);
    return with_type(dout_type, [&](auto x) {
      using X = decltype(x);
      auto* kernel = rows_aligned(dout, ldd, sizeof(X), 16) ? k_embed_few<X, true> : k_embed_few<X, false>;
      kernel<<<unsigned(f.n_sum + a.n_fill), SUM_TPB, 0, st>>>(static_cast<const X*>(dout), f);
      return cuda_ok();
    });
  }
  char* base = static_cast<char*>(workspace);
  SortArgs s;
  s.ids = ids; s.T = T; s.V = V; s.pad_id = pad_id; s.nb_log = p.nb_log; s.bins = int(p.bins);
  s.perm = reinterpret_cast<int32_t*>(base + p.perm);
  s.row = reinterpret_cast<int32_t*>(base + p.row);
  s.start = reinterpret_cast<int32_t*>(base + p.start);
  s.valid = reinterpret_cast<int32_t*>(base + p.valid);
  s.ticket = reinterpret_cast<uint32_t*>(base + p.ticket);
  s.n_ticket = 2 * items;
  const size_t smem = sizeof(SortSmem) + size_t(SORT_WARPS) * p.bins * 4;
  auto* sort = id_type == MV_I32 ? k_embed_sort<int32_t> : k_embed_sort<int64_t>;
  static SmemLimit sort_limit[2];
  if (!allow_smem(sort, int(smem), &sort_limit[id_type == MV_I32])) return MV_ERR_CUDA;
  sort<<<1u << p.nb_log, SORT_TPB, smem, st>>>(s);
  a.perm = s.perm; a.row = s.row; a.start = s.start; a.valid = s.valid; a.ticket = s.ticket;
  a.part = reinterpret_cast<float*>(base + p.part);
  return with_type(dout_type, [&](auto x) {
    using X = decltype(x);
    const bool vec = rows_aligned(dout, ldd, sizeof(X), 16);
    auto* kernel = p.piece == 32 ? (vec ? k_embed_sum<X, true, 32> : k_embed_sum<X, false, 32>)
                                 : (vec ? k_embed_sum<X, true, 8> : k_embed_sum<X, false, 8>);
    const int ring = (p.piece < RING ? p.piece : RING) * SUM_TPB * 16;
    static SmemLimit sum_limit[4];     // (per type of dout)
    if (!allow_smem(kernel, ring, &sum_limit[2 * vec + (p.piece == 32)])) return int(MV_ERR_CUDA);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(n_sum + a.n_fill));
    cfg.blockDim = dim3(SUM_TPB);
    cfg.dynamicSmemBytes = ring;
    cfg.stream = st;
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    const bool ok = cudaLaunchKernelEx(&cfg, kernel, static_cast<const X*>(dout), a) == cudaSuccess;
    return cuda_ok() == MV_OK && ok ? int(MV_OK) : int(MV_ERR_CUDA);
  });
}

}  // extern "C"
