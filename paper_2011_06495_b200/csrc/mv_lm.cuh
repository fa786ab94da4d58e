// mv_lm.cuh -- what the kernels of include/mv_lm.h share: element types, loads and argument checks.
#pragma once
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <mutex>

#include "../../include/mv_sparse.h"
#include "../../include/mv_lm.h"

namespace {

inline bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline int cuda_ok() { return cudaGetLastError() == cudaSuccess ? MV_OK : MV_ERR_CUDA; }

inline bool is_value_type(int t) { return t == MV_F32 || t == MV_BF16 || t == MV_F16; }
inline bool is_id_type(int t) { return t == MV_I32 || t == MV_I64; }
inline int type_size(int t) { return t == MV_F32 || t == MV_I32 ? 4 : t == MV_I64 ? 8 : 2; }

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }

template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }

// id i of an id list, as a row index; -1 for anything outside [0, V)
__device__ __forceinline__ int64_t load_id(const void* ids, int id_type, int64_t i, int64_t V) {
  int64_t v = id_type == MV_I32 ? int64_t(static_cast<const int32_t*>(ids)[i]) : static_cast<const int64_t*>(ids)[i];
  return v >= 0 && v < V ? v : -1;
}

// Whether two strided matrices (rows of `cols` elements of `size` bytes, `ld` elements apart) share bytes: their spans meet, and
// they are not two windows of columns side by side in rows of one pitch (a single row has the other's).
inline bool share_bytes(const void* p, int64_t rows, int64_t cols, int64_t ld, int size, const void* q, int64_t rows2, int64_t cols2, int64_t ld2,
                        int size2) {
  if (rows < 1 || rows2 < 1) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  if (a >= b + size_t((rows2 - 1) * ld2 + cols2) * size2 || b >= a + size_t((rows - 1) * ld + cols) * size) return false;
  const uintptr_t pitch = rows > 1 ? uintptr_t(ld) * size : uintptr_t(ld2) * size2;
  if ((rows2 > 1 && pitch != uintptr_t(ld2) * size2) || (rows < 2 && rows2 < 2)) return true;
  const uintptr_t to = a <= b ? (b - a) % pitch : (pitch - (a - b) % pitch) % pitch;      // from a row of p on to the next row of q
  return to < uintptr_t(cols) * size || pitch - to < uintptr_t(cols2) * size2;
}

// The same for a vector of n elements beside a matrix; an empty or absent one shares nothing.
inline bool share_vector(const void* v, int64_t n, int size, const void* p, int64_t rows, int64_t cols, int64_t ld, int size2) {
  return v && p && n > 0 && share_bytes(p, rows, cols, ld, size2, v, 1, n, n, size);
}

// Dynamic shared memory that a kernel may use without asking: the limit of 48 KB counts its static shared memory (up to 1 KB here) too.
constexpr size_t SMEM_UNASKED = 47 * 1024;

// Lets a kernel use `bytes` of dynamic shared memory; asked of the driver once per kernel (a static of the caller) and device, by one host
// thread at a time, so that what one was granted is not taken back by another's smaller request.
struct SmemLimit {
  int bytes[64] = {};
  std::mutex asking;
};
template <typename K> bool allow_smem(K* kernel, int bytes, SmemLimit* have) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const std::lock_guard<std::mutex> lock(have->asking);
  if (dev < 64 && have->bytes[dev] >= bytes) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  if (dev < 64) have->bytes[dev] = bytes;
  return true;
}

// Calls f with a value of the element type that a type code names.
template <typename F> int with_type(int t, F&& f) {
  switch (t) {
    case MV_F32: return f(float());
    case MV_BF16: return f(__nv_bfloat16());
    case MV_F16: return f(__half());
    default: return MV_ERR_INVALID_ARG;
  }
}

// The same on the device.
template <typename F> __device__ __forceinline__ void with_type_device(int t, F&& f) {
  if (t == MV_F32) f(float());
  else if (t == MV_BF16) f(__nv_bfloat16());
  else f(__half());
}

}  // namespace
