// Row cache in 4 or 8 bits: rows are quantised as they are written and read back as the values their codes stand for.
// A group is one head of one row (dim values):
//     amax = max |x|,  L = 7 or 127,  scale = fp32(amax * fp32(1 / L)) rounded up to bf16,  r = fp32(1 / scale),
//     code = the integer nearest to the exact product x * r (ties to even),  value = code * scale.
// The scale is rounded up so that |x * r| never passes L by more than fp32's roundings, and no code needs clamping.  It is held
// in 16 bits, as bf16, for its fp32 range: more of its bits would be lost on codes of 8 bits or less, and 2 bytes beside 16 to 128
// of codes cost 2 to 12 % where fp32 would cost 3 to 25 %.  A group below 2^-100 is held as zeros (scale 0) so that 1 / scale
// stays in range; a group with an infinity or a NaN has scale NaN and reads back as NaN, all of it, instead of as wrong numbers.
// The product is rounded to an integer by one fused multiply-add onto 1.5 * 2^23, where fp32's spacing is 1: the exact
// product is rounded once, so codes do not depend on how a quotient was computed.  Codes are stored with an offset (8 or 128), which
// leaves them in the low bits of that sum; a word of them is put together by shifted adds.
//
// Layout: codes [heads][pad * bits / 8 bytes] per row, pad = 32, 64 or 128 values of a head (padding holds code 0), scales bf16 [heads]
// per row, one fp64 time per row; each with a row stride of its own, so that a row can also be one record of a send buffer.
//
// Both kernels are bound by HBM: 8 values per thread, and the rows of four groups in flight per thread.
#include "tgnn_history.cuh"

using namespace tgnn_history;

namespace {

constexpr int THREADS = 256;
constexpr int U = 4;              // groups per thread, loaded together

__device__ __forceinline__ int64_t index_at(const void* idx, int index64, int64_t i) {
  if (!idx) return i;
  return index64 ? __ldg(reinterpret_cast<const long long*>(idx) + i) : (int64_t)__ldg(reinterpret_cast<const int*>(idx) + i);
}

__device__ __forceinline__ float max_nan(float a, float b) {      // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// 8 values of a row from element `e0` on, VB bytes at a time; values at and beyond dim are 0.  VB / sizeof(T) divides dim.
template <typename T, int VB>
__device__ __forceinline__ void load8(const T* row, int e0, int dim, float (&v)[8]) {
  constexpr int VE = VB / (int)sizeof(T);
#pragma unroll
  for (int j = 0; j < 8; j += VE) {
    union { typename Vec<VB>::type w; T x[VE]; } p;
    const bool in = e0 + j < dim;
    if (in) p.w = __ldg(reinterpret_cast<const typename Vec<VB>::type*>(row + e0 + j));
#pragma unroll
    for (int i = 0; i < VE; ++i) v[j + i] = in ? to_float<T>(p.x[i]) : 0.f;
  }
}

template <typename T, int VB>
__device__ __forceinline__ void store8(T* row, int e0, int dim, const float (&v)[8]) {
  constexpr int VE = VB / (int)sizeof(T);
#pragma unroll
  for (int j = 0; j < 8; j += VE) {
    union { typename Vec<VB>::type w; T x[VE]; } p;
#pragma unroll
    for (int i = 0; i < VE; ++i) p.x[i] = from_float<T>(v[j + i]);
    if (e0 + j < dim) *reinterpret_cast<typename Vec<VB>::type*>(row + e0 + j) = p.w;
  }
}

// A group is handled by 2^lg neighbouring lanes (pad / 8 of them); groups are numbered row by row.
template <typename T, int VB, int BITS>
__global__ void __launch_bounds__(THREADS) cache_write_kernel(const CacheView c, const T* __restrict__ rows, int64_t num_rows,
                                                              int64_t row_stride, const void* __restrict__ src,
                                                              const void* __restrict__ dst, int index64, uint32_t groups,
                                                              const double* __restrict__ times, int32_t* status, int lg) {
  const int lanes = 1 << lg, l = threadIdx.x & (lanes - 1);
  const uint32_t g0 = (uint32_t)(((uint64_t)blockIdx.x * (THREADS * U) + threadIdx.x) >> lg);
  float v[U][8];
  int64_t place[U];
  int head[U];
  double when[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t g = g0 + u * (THREADS >> lg);
    place[u] = -1;
    when[u] = 0.0;
    int64_t from = -1;
    head[u] = 0;
    if (g < groups) {
      const uint32_t i = g / (uint32_t)c.heads;
      head[u] = (int)(g - i * (uint32_t)c.heads);
      from = index_at(src, index64, i);
      place[u] = index_at(dst, index64, i);
      if (from < 0 || from >= num_rows) { from = -1; atomicMax(status, 4); }
      if (place[u] < 0 || place[u] >= c.rows) { place[u] = -1; atomicMax(status, 4); }
    }
    if (from >= 0) {
      load8<T, VB>(rows + from * row_stride + (int64_t)head[u] * c.dim, 8 * l, c.dim, v[u]);
      if (times && head[u] == 0 && l == 0) when[u] = __ldg(times + from);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[u][j] = 0.f;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float amax = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) amax = max_nan(amax, fabsf(v[u][j]));
    for (int o = lanes >> 1; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(FULL, amax, o));
    const bool bad = !(amax <= 3.4028234e38f);
    float s = __uint_as_float((__float_as_uint(__fmul_rn(amax, BITS == 4 ? 1.f / 7.f : 1.f / 127.f)) + 0xffffu) & 0xffff0000u);
    if (amax < 7.8886091e-31f) s = 0.f;                                   // 2^-100
    const float r = s > 0.f ? __frcp_rn(s) : 0.f;
    uint32_t w[BITS == 4 ? 1 : 2];
    // float bits of 1.5 * 2^23 + offset + code, added up with shifts; the fixed part of the sum is taken off at the end
    constexpr float kMagic = 12582912.f + (BITS == 4 ? 8.f : 128.f);
    constexpr int PER = BITS == 4 ? 8 : 4;
#pragma unroll
    for (int q = 0; q < 8 / PER; ++q) {
      uint32_t acc = 0, fixed = 0;
#pragma unroll
      for (int j = PER - 1; j >= 0; --j) {
        acc = (acc << BITS) + __float_as_uint(fmaf(v[u][q * PER + j], r, kMagic));
        fixed = (fixed << BITS) + 0x4b400000u;
      }
      w[q] = bad ? (BITS == 4 ? 0x88888888u : 0x80808080u) : acc - fixed;
    }
    if (place[u] >= 0) {
      uint8_t* to = c.codes + place[u] * c.code_stride + (int64_t)head[u] * c.code_bytes;
      if (BITS == 4) reinterpret_cast<uint32_t*>(to)[l] = w[0];
      else reinterpret_cast<uint2*>(to)[l] = make_uint2(w[0], w[BITS == 4 ? 0 : 1]);
      if (l == 0) {
        const uint16_t bits = bad ? (uint16_t)0x7fc0u : (uint16_t)(__float_as_uint(s) >> 16);
        *reinterpret_cast<uint16_t*>(c.scales + place[u] * c.scale_stride + 2 * head[u]) = bits;
        if (times && c.times && head[u] == 0) *reinterpret_cast<double*>(c.times + place[u] * c.time_stride) = when[u];
      }
    }
  }
}

template <typename T, int VB, int BITS>
__global__ void __launch_bounds__(THREADS) cache_read_kernel(const CacheView c, T* __restrict__ rows, int64_t num_rows,
                                                             int64_t row_stride, const void* __restrict__ src,
                                                             const void* __restrict__ dst, int index64, uint32_t groups,
                                                             double* __restrict__ times, int32_t* status, int lg) {
  const int lanes = 1 << lg, l = threadIdx.x & (lanes - 1);
  const uint32_t g0 = (uint32_t)(((uint64_t)blockIdx.x * (THREADS * U) + threadIdx.x) >> lg);
  uint32_t w[U][2];
  uint16_t sb[U];
  double when[U];
  int64_t to[U];
  int head[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t g = g0 + u * (THREADS >> lg);
    to[u] = -1;
    head[u] = 0;
    sb[u] = 0;
    when[u] = 0.0;
    w[u][0] = w[u][1] = 0;
    if (g < groups) {
      const uint32_t i = g / (uint32_t)c.heads;
      head[u] = (int)(g - i * (uint32_t)c.heads);
      const int64_t place = index_at(src, index64, i);
      to[u] = index_at(dst, index64, i);
      if (to[u] < 0 || to[u] >= num_rows) { to[u] = -1; atomicMax(status, 4); }
      if (place < 0 || place >= c.rows) {
        atomicMax(status, 4);                                             // reads as zeros
      } else {
        const uint8_t* from = c.codes + place * c.code_stride + (int64_t)head[u] * c.code_bytes;
        if (BITS == 4) {
          w[u][0] = __ldg(reinterpret_cast<const uint32_t*>(from) + l);
        } else {
          const uint2 p = __ldg(reinterpret_cast<const uint2*>(from) + l);
          w[u][0] = p.x;
          w[u][1] = p.y;
        }
        sb[u] = __ldg(reinterpret_cast<const uint16_t*>(c.scales + place * c.scale_stride + 2 * head[u]));
        if (times && c.times && head[u] == 0 && l == 0) when[u] = __ldg(reinterpret_cast<const double*>(c.times + place * c.time_stride));
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (to[u] >= 0) {
      const float s = __uint_as_float((uint32_t)sb[u] << 16);
      float v[8];
      // a code under fp32's exponent for 2^23 reads as 2^23 + offset + code
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t code = BITS == 4 ? (w[u][0] >> (4 * j)) & 0xfu : (w[u][j >> 2] >> (8 * (j & 3))) & 0xffu;
        v[j] = (__uint_as_float(0x4b000000u | code) - (8388608.f + (BITS == 4 ? 8.f : 128.f))) * s;
      }
      store8<T, VB>(rows + to[u] * row_stride + (int64_t)head[u] * c.dim, 8 * l, c.dim, v);
      if (times && c.times && head[u] == 0 && l == 0) times[to[u]] = when[u];
    }
  }
}

struct Args {
  CacheView c;
  void* rows;
  int64_t num_rows, row_stride;
  const void *src, *dst;
  int index64;
  uint32_t groups;
  double* times;
  int32_t* status;
  int lg;
  cudaStream_t s;
};

template <bool WRITE, typename T, int VB, int BITS>
void launch(const Args& a) {
  const uint64_t threads = (uint64_t)a.groups << a.lg;
  const unsigned grid = (unsigned)((threads + THREADS * U - 1) / (THREADS * U));
  if (WRITE)
    cache_write_kernel<T, VB, BITS><<<grid, THREADS, 0, a.s>>>(a.c, (const T*)a.rows, a.num_rows, a.row_stride, a.src, a.dst,
                                                               a.index64, a.groups, a.times, a.status, a.lg);
  else
    cache_read_kernel<T, VB, BITS><<<grid, THREADS, 0, a.s>>>(a.c, (T*)a.rows, a.num_rows, a.row_stride, a.src, a.dst, a.index64,
                                                              a.groups, a.times, a.status, a.lg);
}

// Rows move in words of 16 bytes where base, row stride and head all start on one, else of 8 (heads of 50 in fp32), 4 (heads of 50
// in 16 bits) or single values.
template <bool WRITE, typename T, int BITS>
void launch_aligned(const Args& a) {
  const uint64_t at = (uint64_t)(uintptr_t)a.rows | (uint64_t)(a.row_stride * (int64_t)sizeof(T)) | (uint64_t)(a.c.dim * (int)sizeof(T));
  if ((at & 15) == 0) launch<WRITE, T, 16, BITS>(a);
  else if (sizeof(T) == 4 && (at & 7) == 0) launch<WRITE, T, 8, BITS>(a);
  else if ((at & 3) == 0) launch<WRITE, T, 4, BITS>(a);
  else launch<WRITE, T, sizeof(T), BITS>(a);
}

template <bool WRITE>
int run(const char* who, const tgnn_cache* cache, void* rows, int dtype, int64_t num_rows, int64_t row_stride, const void* src,
        const void* dst, int index_bits, int64_t n, double* times, int32_t* status, void* stream, char* err, int64_t size) {
  Args a;
  const int rc = check_cache(who, "cache", cache, &a.c, err, size);
  if (rc) return rc;
  if (!known_dtype(dtype)) return fail(err, size, TGNN_EINVAL, "%s: unknown row type %d", who, dtype);
  if ((src || dst) && index_bits != 32 && index_bits != 64)
    return fail(err, size, TGNN_EINVAL, "%s: indices have 32 or 64 bits, not %d", who, index_bits);
  if (num_rows < 0 || n < 0 || row_stride < (int64_t)a.c.heads * a.c.dim)
    return fail(err, size, TGNN_EINVAL, "%s: size out of range (a row holds heads * dim values)", who);
  if (n > 0x7fffffff / a.c.heads) return fail(err, size, TGNN_ECAPACITY, "%s: n * heads beyond int32", who);
  if (!status || (n > 0 && num_rows > 0 && !rows)) return fail(err, size, TGNN_EINVAL, "%s: null pointer", who);
  if (times && n > 0 && !a.c.times) return fail(err, size, TGNN_EINVAL, "%s: times given, but the cache holds none", who);
  const int idx = index_bits == 64 ? 7 : 3;
  if (((uintptr_t)rows & (elem_bytes(dtype) - 1)) || (((uintptr_t)src | (uintptr_t)dst) & idx) || ((uintptr_t)times & 7) ||
      ((uintptr_t)status & 3))
    return fail(err, size, TGNN_EINVAL, "%s: a pointer is not aligned to its element", who);
  if (n == 0) return TGNN_OK;
  a.rows = rows;
  a.num_rows = num_rows;
  a.row_stride = row_stride;
  a.src = src;
  a.dst = dst;
  a.index64 = index_bits == 64;
  a.groups = (uint32_t)(n * a.c.heads);
  a.times = times;
  a.status = status;
  a.s = (cudaStream_t)stream;
  const int pad = padded_dim(a.c.dim);
  a.lg = pad == 32 ? 2 : pad == 64 ? 3 : 4;
  const bool four = a.c.bits == 4;
  if (dtype == TGNN_F32) four ? launch_aligned<WRITE, float, 4>(a) : launch_aligned<WRITE, float, 8>(a);
  else if (dtype == TGNN_BF16) four ? launch_aligned<WRITE, __nv_bfloat16, 4>(a) : launch_aligned<WRITE, __nv_bfloat16, 8>(a);
  else four ? launch_aligned<WRITE, __half, 4>(a) : launch_aligned<WRITE, __half, 8>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return fail(err, size, TGNN_ECUDA, "%s: %s", who, cudaGetErrorString(e));
  return TGNN_OK;
}

}  // namespace

extern "C" {

int64_t tgnn_cache_code_bytes(int dim, int bits) {
  if (dim < 1 || dim > 128 || (bits != 4 && bits != 8)) return -1;
  return padded_dim(dim) * bits / 8;
}

int tgnn_cache_write(const tgnn_cache* cache_host, const void* rows, int dtype, int64_t num_rows, int64_t row_stride, const void* src,
                     const void* dst, int index_bits, int64_t n, const double* times, int32_t* status, void* stream, char* err_host,
                     int64_t err_size) {
  return run<true>("tgnn_cache_write", cache_host, const_cast<void*>(rows), dtype, num_rows, row_stride, src, dst, index_bits, n,
                   const_cast<double*>(times), status, stream, err_host, err_size);
}

int tgnn_cache_read(const tgnn_cache* cache_host, void* rows, int dtype, int64_t num_rows, int64_t row_stride, const void* src,
                    const void* dst, int index_bits, int64_t n, double* times, int32_t* status, void* stream, char* err_host,
                    int64_t err_size) {
  return run<false>("tgnn_cache_read", cache_host, rows, dtype, num_rows, row_stride, src, dst, index_bits, n, times, status, stream,
                    err_host, err_size);
}

}  // extern "C"
