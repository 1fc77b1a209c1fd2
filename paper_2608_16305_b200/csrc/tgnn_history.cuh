// What the history operators share (row cache, attention over it, slot attention): error texts, row types, the time
// buckets and the view of a row cache.
#pragma once
#include <atomic>
#include <cstdarg>
#include <cstdio>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/tgnn.h"

namespace tgnn_history {

constexpr unsigned FULL = 0xffffffffu;
constexpr int kMaxBuckets = 128;
constexpr float kLog2e = 1.4426950408889634f;

inline int fail(char* err, int64_t size, int code, const char* fmt, ...) {
  if (err && size > 0) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(err, (size_t)size, fmt, ap);
    va_end(ap);
  }
  return code;
}

inline int elem_bytes(int dtype) { return dtype == TGNN_F32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == TGNN_F32 || dtype == TGNN_BF16 || dtype == TGNN_F16; }

// Values that a head's codes are padded to: the readers' tiles of 32, 64 or 128.
inline int padded_dim(int dim) { return dim <= 32 ? 32 : dim <= 64 ? 64 : 128; }

// Multiprocessors of the current device (asked for once per device, by any thread; the answer cannot change).
inline int num_sms() {
  static std::atomic<int> cached[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 148;
  if (dev >= 0 && dev < 64 && (n = cached[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = 148;
  if (dev >= 0 && dev < 64) cached[dev].store(n, std::memory_order_relaxed);
  return n;
}

template <typename T>
__device__ __forceinline__ float to_float(T x);
template <>
__device__ __forceinline__ float to_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float to_float<__half>(__half x) { return __half2float(x); }
// One rounding to the row type, to nearest even.
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// The row types' largest finite values, and how far a finite row's values may pass them: a cache's scale is rounded up to bf16, so the
// largest code times the scale lies up to 2^-7 above the group's largest magnitude.  fp16 has numbers of fp32 beyond that, which convert to
// infinity; of fp32 and bf16 nothing finite is further out.
template <typename T>
struct Range { static constexpr float most = 3.40282347e38f, edge = INFINITY; };
template <>
struct Range<__nv_bfloat16> { static constexpr float most = 3.38953139e38f, edge = INFINITY; };
template <>
struct Range<__half> { static constexpr float most = 65504.f, edge = 66016.f; };   // 65504 (1 + 2^-7) is 66015.75
// x, or the largest finite value where x is past it by no more than that; NaN stays.
template <typename T>
__device__ __forceinline__ float within(float x) {
  return fabsf(x) > Range<T>::most && fabsf(x) <= Range<T>::edge ? copysignf(Range<T>::most, x) : x;
}

// Words of VB bytes.
template <int VB>
struct Vec;
template <>
struct Vec<16> { typedef uint4 type; };
template <>
struct Vec<8> { typedef uint2 type; };
template <>
struct Vec<4> { typedef uint32_t type; };
template <>
struct Vec<2> { typedef uint16_t type; };

// 2^x, relative error 2^-22; results below 2^-126 are 0.
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// 1 / x, relative error 2^-23, for normal x (and NaN).
__device__ __forceinline__ float rcp_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Bucket of a time difference: how many of the n ascending bounds are <= dt.  The comparisons are in fp64, so a difference
// on a bound lands where the definition says; NaN is above no bound.
// In shared memory the bounds lie behind a -infinity and before +infinities: s[i] is bound i - 1, s[kMaxBuckets] the last.
__device__ __forceinline__ void stage_bounds(double* s, const double* bounds, int n, int thread, int threads) {
  for (int i = thread; i <= kMaxBuckets; i += threads) s[i] = i == 0 ? -INFINITY : i <= n ? bounds[i - 1] : INFINITY;
}
// Halving without branches: the largest i <= n with bounds 1 to i <= dt.
__device__ __forceinline__ int bucket_of(const double* s, int n, double dt) {
  int b = 0;
#pragma unroll
  for (int step = kMaxBuckets / 2; step > 0; step >>= 1)
    if (s[b + step] <= dt) b += step;
  return min(b, n);                                            // dt = +infinity passes the padding too
}
// The same for all lanes of a warp, where most of them share the bucket b of the last entry that they looked at.
__device__ __forceinline__ int bucket_near(const double* s, int n, double dt, int b) {
  if (!__all_sync(FULL, s[b] <= dt && dt < s[b + 1])) b = bucket_of(s, n, dt);
  return b;
}

// A row cache as the kernels see it (tgnn_cache with the codes' size).
struct CacheView {
  uint8_t* codes;
  uint8_t* scales;
  uint8_t* times;
  int64_t rows, code_stride, scale_stride, time_stride;
  int heads, dim, bits, code_bytes;      // code_bytes: of one head in a row
};

// Checks a cache description and fills its view; the entry point's name goes into the message.
inline int check_cache(const char* who, const char* which, const tgnn_cache* c, CacheView* v, char* err, int64_t size) {
  if (!c) return fail(err, size, TGNN_EINVAL, "%s: %s is null", who, which);
  if (c->bits != 4 && c->bits != 8) return fail(err, size, TGNN_EINVAL, "%s: %s has %d bits (4 or 8)", who, which, c->bits);
  if (c->dim < 1 || c->dim > 128 || c->heads < 1 || c->heads > 1024 || c->rows < 0)
    return fail(err, size, TGNN_EINVAL, "%s: %s: size out of range (dim 1 to 128, heads 1 to 1024)", who, which);
  const int gb = padded_dim(c->dim) * c->bits / 8;
  if (c->rows > 0 && (!c->codes || !c->scales)) return fail(err, size, TGNN_EINVAL, "%s: %s: null pointer", who, which);
  if (((uintptr_t)c->codes & 15) || (c->code_stride & 15) || ((uintptr_t)c->scales & 1) || (c->scale_stride & 1) ||
      ((uintptr_t)c->times & 7) || (c->times && (c->time_stride & 7)))
    return fail(err, size, TGNN_EINVAL, "%s: %s: codes must be 16-byte, scales 2-byte and times 8-byte aligned, strides too", who, which);
  if (c->code_stride < (int64_t)c->heads * gb || c->scale_stride < 2 * (int64_t)c->heads || (c->times && c->time_stride < 8))
    return fail(err, size, TGNN_EINVAL, "%s: %s: stride shorter than a row", who, which);
  if (c->code_stride > 0x7fffffff || c->scale_stride > 0x7fffffff || (c->times && c->time_stride > 0x7fffffff))
    return fail(err, size, TGNN_ECAPACITY, "%s: %s: stride beyond int32", who, which);
  v->codes = (uint8_t*)c->codes;
  v->scales = (uint8_t*)c->scales;
  v->times = (uint8_t*)c->times;
  v->rows = c->rows;
  v->code_stride = c->code_stride;
  v->scale_stride = c->scale_stride;
  v->time_stride = c->time_stride;
  v->heads = c->heads;
  v->dim = c->dim;
  v->bits = c->bits;
  v->code_bytes = gb;
  return TGNN_OK;
}

}  // namespace tgnn_history
