// Row cache in 4 or 8 bits: rows are quantised as they are written and read back as the values their codes stand for.
// A group is one head of one row (dim values):
//     amax = max |x|,  L = 7 or 127,  scale = fp32(amax * fp32(1 / L)) rounded up to bf16,  r = fp32(1 / scale),
//     code = the integer nearest to the exact product x * r (ties to even),  value = code * scale.
// The scale is rounded up so that |x * r| never passes L by more than fp32's roundings, and no code needs clamping.  It is held
// in 16 bits, as bf16, for its fp32 range: more of its bits would be lost on codes of 8 bits or less, and 2 bytes beside 16 to 128
// of codes cost 2 to 12 % where fp32 would cost 3 to 25 %.  A group below 2^-100 is held as zeros (scale 0) so that 1 / scale
// stays in range; a group with an infinity or a NaN has scale NaN and reads back as NaN, all of it, instead of as wrong numbers.
// (Read back, the largest code may then lie past the row type's largest finite value, by 2^-7 of it at most: it is held at that value, so that
// finite rows stay finite.  A wider row read as fp16 is infinite beyond that, as by any conversion.)
// The product is rounded to an integer by one fused multiply-add onto 1.5 * 2^23, where fp32's spacing is 1: the exact
// product is rounded once, so codes do not depend on how a quotient was computed.  Codes are stored with an offset (8 or 128), which
// leaves them in the low bits of that sum; a word of them is put together by shifted adds.
//
// Layout: codes [heads][pad * bits / 8 bytes] per row, pad = 32, 64 or 128 values of a head (padding holds code 0), scales bf16 [heads]
// per row, one fp64 time per row; each with a row stride of its own, so that a row can also be one record of a send buffer.
//
// Both kernels are bound by HBM.  2 to 8 neighbouring lanes take a row, head after head, two heads at a time where there are two.  A lane
// takes two pieces of 8 values of a head, half a head apart, so that the lanes of a row move whole sectors; the index arithmetic of
// a row is done once.
//
// Measured on a B200, a million rows of 4 x 64 in bf16 at random places, in 4 bits: written in 141 us (4.8 TB/s of DRAM), read back in
// 138 us (4.7); a copy of whole tables reaches 6.5.
#include "tgnn_history.cuh"

using namespace tgnn_history;

namespace {

constexpr int THREADS = 256;

struct Move {
  CacheView c;
  int64_t num_rows;
  uint32_t row_bytes;             // of a table row to the next
  const void *src, *dst;
  int index64;
  uint32_t n;
  double* times;
  int32_t* status;
  int lg;                         // 2^lg lanes per row: pad / 16
};

__device__ __forceinline__ int64_t index_at(const void* idx, int index64, uint32_t i) {
  if (!idx) return i;
  return index64 ? __ldg(reinterpret_cast<const long long*>(idx) + i) : (int64_t)__ldg(reinterpret_cast<const int*>(idx) + i);
}

// The table row and the cache row of list entry i, negative where an index lies outside (recorded) or the list has ended.
struct Where {
  int64_t row, place;
};
template <bool WRITE>
__device__ __forceinline__ Where find(const Move& a, uint64_t i) {
  Where w = {-1, -1};
  if (i < a.n) {
    w.row = index_at(WRITE ? a.src : a.dst, a.index64, (uint32_t)i);
    w.place = index_at(WRITE ? a.dst : a.src, a.index64, (uint32_t)i);
    const bool out_row = (uint64_t)w.row >= (uint64_t)a.num_rows, out_place = (uint64_t)w.place >= (uint64_t)a.c.rows;
    if (out_row | out_place) {
      atomicMax(a.status, 4);
      if (out_row) w.row = -1;
      if (out_place) w.place = -1;
    }
  }
  return w;
}

__device__ __forceinline__ float max_nan(float a, float b) {      // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// 8 values of a row from element `e0` on, VB bytes at a time, as they are in memory; values at and beyond dim are 0.  VB / sizeof(T)
// divides dim.
template <typename T, int VB>
struct Eight {
  static constexpr int VE = VB / (int)sizeof(T);
  union Word { typename Vec<VB>::type w; T x[VE]; };
  Word p[8 / VE];
  __device__ __forceinline__ void load(const T* row, int e0, int dim, bool on) {
#pragma unroll
    for (int j = 0; j < 8 / VE; ++j) {
      p[j].w = typename Vec<VB>::type();
      if (on && e0 + j * VE < dim) p[j].w = __ldg(reinterpret_cast<const typename Vec<VB>::type*>(row + e0 + j * VE));
    }
  }
  __device__ __forceinline__ float at(int j) const { return to_float<T>(p[j / VE].x[j % VE]); }
};

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

// The group's scale (the bits of a bf16) from its largest magnitude, and the codes of two times 8 of its values.
template <int BITS>
__device__ __forceinline__ uint16_t quantise(float amax, const float (*v)[8], uint32_t (*code)[BITS == 4 ? 1 : 2]) {
  const bool bad = !(amax <= 3.4028234e38f);
  float s = __uint_as_float((__float_as_uint(__fmul_rn(amax, BITS == 4 ? 1.f / 7.f : 1.f / 127.f)) + 0xffffu) & 0xffff0000u);
  if (amax < 7.8886091e-31f) s = 0.f;                                     // 2^-100
  const float r = s > 0.f ? __frcp_rn(s) : 0.f;
  // float bits of 1.5 * 2^23 + offset + code, added up with shifts; the fixed part of the sum is taken off at the end
  constexpr float kMagic = 12582912.f + (BITS == 4 ? 8.f : 128.f);
  constexpr int PER = BITS == 4 ? 8 : 4, WORDS = 8 / PER;
#pragma unroll
  for (int p = 0; p < 2; ++p) {
#pragma unroll
    for (int q = 0; q < WORDS; ++q) {
      uint32_t acc = 0, fixed = 0;
#pragma unroll
      for (int j = PER - 1; j >= 0; --j) {
        acc = (acc << BITS) + __float_as_uint(fmaf(v[p][q * PER + j], r, kMagic));
        fixed = (fixed << BITS) + 0x4b400000u;
      }
      code[p][q] = bad ? (BITS == 4 ? 0x88888888u : 0x80808080u) : acc - fixed;
    }
  }
  return bad ? (uint16_t)0x7fc0u : (uint16_t)(__float_as_uint(s) >> 16);
}

// The 8 values of codes, for rows of T: a code under fp32's exponent for 2^23 reads as 2^23 + offset + code.
template <typename T, int BITS>
__device__ __forceinline__ void values(const uint32_t (&code)[BITS == 4 ? 1 : 2], float s, float (&v)[8]) {
  constexpr int PER = BITS == 4 ? 8 : 4;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t x = (code[j / PER] >> (BITS * (j % PER))) & (BITS == 4 ? 0xfu : 0xffu);
    v[j] = (__uint_as_float(0x4b000000u | x) - (8388608.f + (BITS == 4 ? 8.f : 128.f))) * s;
  }
  if (s * (BITS == 4 ? 7.f : 127.f) > Range<T>::most) {         // (NaN is not)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = within<T>(v[j]);
  }
}

// U heads of a row at a time: 2, or 1 for rows of one head.  (A million rows of 4 x 64 in bf16 in 4 bits, written and read: 298 us; four at
// a time, whose registers leave half the warps, 312 to 340 us.)
template <typename T, int VB, int BITS, int U>
__global__ void __launch_bounds__(THREADS) cache_write_kernel(const Move a, const T* __restrict__ rows) {
  const int lanes = 1 << a.lg, l = threadIdx.x & (lanes - 1);
  const Where w = find<true>(a, ((uint64_t)blockIdx.x * THREADS + threadIdx.x) >> a.lg);
  const T* row = reinterpret_cast<const T*>(reinterpret_cast<const uint8_t*>(rows) + (uint64_t)(uint32_t)w.row * a.row_bytes);
  const uint64_t place = (uint32_t)w.place;
  uint8_t* to = a.c.codes + place * (uint32_t)a.c.code_stride;
  uint16_t* scales = reinterpret_cast<uint16_t*>(a.c.scales + place * (uint32_t)a.c.scale_stride);
  if (a.times && l == 0 && w.place >= 0)
    *reinterpret_cast<double*>(a.c.times + place * (uint32_t)a.c.time_stride) = w.row >= 0 ? __ldg(a.times + w.row) : 0.0;
  for (int h = 0; h < a.c.heads; h += U) {
    Eight<T, VB> raw[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool on = w.row >= 0 && h + u < a.c.heads;
      raw[u][0].load(row + u * a.c.dim, 8 * l, a.c.dim, on);
      raw[u][1].load(row + u * a.c.dim, 8 * (l + lanes), a.c.dim, on);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[2][8];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j >> 3][j & 7] = raw[u][j >> 3].at(j & 7);
      float amax = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = max_nan(amax, max_nan(fabsf(v[0][j]), fabsf(v[1][j])));
      amax = max_nan(amax, __shfl_xor_sync(FULL, amax, 1));
      if (lanes > 2) amax = max_nan(amax, __shfl_xor_sync(FULL, amax, 2));
      if (lanes > 4) amax = max_nan(amax, __shfl_xor_sync(FULL, amax, 4));
      constexpr int WORDS = BITS == 4 ? 1 : 2;
      uint32_t code[2][WORDS];
      const uint16_t sb = quantise<BITS>(amax, v, code);
      if (w.place >= 0 && h + u < a.c.heads) {
        if constexpr (BITS == 4) {
          reinterpret_cast<uint32_t*>(to + u * a.c.code_bytes)[l] = code[0][0];
          reinterpret_cast<uint32_t*>(to + u * a.c.code_bytes)[l + lanes] = code[1][0];
        } else {
          reinterpret_cast<uint2*>(to + u * a.c.code_bytes)[l] = make_uint2(code[0][0], code[0][1]);
          reinterpret_cast<uint2*>(to + u * a.c.code_bytes)[l + lanes] = make_uint2(code[1][0], code[1][1]);
        }
        if (l == 0) scales[h + u] = sb;
      }
    }
    row += U * a.c.dim;
    to += U * a.c.code_bytes;
  }
}

// Eight blocks to an SM where a row moves in 16-byte words: the branch for the end of the type's range, hardly ever taken, would cost registers (a million
// rows of 4 x 64 in fp32 from 8 bits: 318 us, 343 without that branch and without the bound).  Narrower words are better off with registers for
// all their addresses than with more warps (400 000 rows of 8 x 50 in bf16 from 4 bits: 223 us, 340 with the bound).
template <typename T, int VB, int BITS, int U>
__global__ void __launch_bounds__(THREADS, VB == 16 ? 8 : 1) cache_read_kernel(const Move a, T* __restrict__ rows) {
  const int lanes = 1 << a.lg, l = threadIdx.x & (lanes - 1);
  constexpr int PER = BITS == 4 ? 8 : 4, WORDS = 8 / PER;
  const Where w = find<false>(a, ((uint64_t)blockIdx.x * THREADS + threadIdx.x) >> a.lg);
  if (w.row < 0) return;
  T* row = reinterpret_cast<T*>(reinterpret_cast<uint8_t*>(rows) + (uint64_t)(uint32_t)w.row * a.row_bytes);
  const uint64_t place = (uint32_t)w.place;
  const uint8_t* from = a.c.codes + place * (uint32_t)a.c.code_stride;
  const uint16_t* scales = reinterpret_cast<const uint16_t*>(a.c.scales + place * (uint32_t)a.c.scale_stride);
  if (a.times && l == 0)
    a.times[w.row] = w.place >= 0 ? __ldg(reinterpret_cast<const double*>(a.c.times + place * (uint32_t)a.c.time_stride)) : 0.0;
  for (int h = 0; h < a.c.heads; h += U) {
    uint32_t code[U][2][WORDS], sb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      sb[u] = 0;                                               // an index outside reads as zeros: scale 0
#pragma unroll
      for (int q = 0; q < WORDS; ++q) code[u][0][q] = code[u][1][q] = 0;
      if (w.place >= 0 && h + u < a.c.heads) {
        if constexpr (BITS == 4) {
          code[u][0][0] = __ldg(reinterpret_cast<const uint32_t*>(from + u * a.c.code_bytes) + l);
          code[u][1][0] = __ldg(reinterpret_cast<const uint32_t*>(from + u * a.c.code_bytes) + l + lanes);
        } else {
          const uint2 p = __ldg(reinterpret_cast<const uint2*>(from + u * a.c.code_bytes) + l);
          const uint2 q = __ldg(reinterpret_cast<const uint2*>(from + u * a.c.code_bytes) + l + lanes);
          code[u][0][0] = p.x;
          code[u][0][1] = p.y;
          code[u][1][0] = q.x;
          code[u][1][1] = q.y;
        }
        sb[u] = __ldg(scales + h + u);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h + u >= a.c.heads) break;
      const float s = __uint_as_float(sb[u] << 16);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        float v[8];
        values<T, BITS>(code[u][p], s, v);
        store8<T, VB>(row + u * a.c.dim, 8 * (l + p * lanes), a.c.dim, v);
      }
    }
    row += U * a.c.dim;
    from += U * a.c.code_bytes;
  }
}

// Reading into rows whose heads start on no word of several values (odd heads, odd bases): written value by value in the order of the codes, the
// lanes of a warp would touch a sector each.  Here a warp moves 32 / lanes whole groups (heads of rows, numbered row by row): 8 values per lane as above
// go to shared memory, as fp32, and from there in words of VB bytes that lie side by side.  A group's
// place in shared memory is a multiple of 8 and one long, which spreads the lanes' accesses over the banks.
template <typename T, int VB, int BITS>
__global__ void __launch_bounds__(THREADS) cache_read_narrow_kernel(const Move a, T* __restrict__ rows) {
  constexpr int VE = VB / (int)sizeof(T), N = 8 / VE, WORDS = BITS == 4 ? 1 : 2;
  typedef typename Vec<VB>::type W;
  union Word { W w; T x[VE]; };
  __shared__ float s_values[THREADS / 32][256 + 8];
  const int lane = threadIdx.x & 31, lg = a.lg + 1, lanes = 1 << lg, count = 32 >> lg, ld = 8 * lanes + 1;
  float* mine = s_values[threadIdx.x >> 5];
  const uint64_t g0 = ((uint64_t)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5)) * count, g = g0 + lane;
  // lane i < count: where group g0 + i lies
  Where w = {-1, -1};
  int head = 0;
  if (lane < count && g < (uint64_t)a.n * a.c.heads) {
    const uint32_t i = (uint32_t)g / (uint32_t)a.c.heads;
    head = (int)((uint32_t)g - i * (uint32_t)a.c.heads);
    w = find<false>(a, i);
  }
  if (a.times && head == 0 && w.row >= 0)
    a.times[w.row] = w.place >= 0 ? __ldg(reinterpret_cast<const double*>(a.c.times + (uint64_t)(uint32_t)w.place * (uint32_t)a.c.time_stride)) : 0.0;
  const int64_t row_at = w.row < 0 ? -1 : (int64_t)((uint64_t)(uint32_t)w.row * a.row_bytes) + (int64_t)head * a.c.dim * (int)sizeof(T);
  const int per = a.c.dim / VE, magic = (65536 + per - 1) / per;     // word x of the warp belongs to group (x * magic) >> 16: exact below 256
  const int own = lane >> lg, l = lane & (lanes - 1);                // the lane's group and its 8 values there
  const int64_t place = __shfl_sync(FULL, w.place, own);
  const int own_head = __shfl_sync(FULL, head, own);
  uint32_t code[WORDS] = {};
  uint32_t sb = 0;
  if (place >= 0) {
    const uint8_t* codes = a.c.codes + (uint64_t)place * (uint32_t)a.c.code_stride + own_head * a.c.code_bytes;
    if constexpr (BITS == 4) {
      code[0] = __ldg(reinterpret_cast<const uint32_t*>(codes) + l);
    } else {
      const uint2 p = __ldg(reinterpret_cast<const uint2*>(codes) + l);
      code[0] = p.x;
      code[WORDS - 1] = p.y;
    }
    sb = __ldg(reinterpret_cast<const uint16_t*>(a.c.scales + (uint64_t)place * (uint32_t)a.c.scale_stride) + own_head);
  }
  float v[8];
  values<T, BITS>(code, __uint_as_float(sb << 16), v);
#pragma unroll
  for (int j = 0; j < 8; ++j) mine[own * ld + 8 * l + j] = v[j];
  __syncwarp();
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int x = lane + 32 * j, grp = min((x * magic) >> 16, count - 1), off = x - grp * per;
    const int64_t to = __shfl_sync(FULL, row_at, grp);
    if (off < per && to >= 0) {
      Word out;
#pragma unroll
      for (int e = 0; e < VE; ++e) out.x[e] = from_float<T>(mine[grp * ld + off * VE + e]);
      reinterpret_cast<W*>(reinterpret_cast<uint8_t*>(rows) + to)[off] = out.w;
    }
  }
}

template <bool WRITE, typename T, int VB, int BITS, int U>
void launch_heads(const Move& a, void* rows, cudaStream_t s) {
  const unsigned grid = (unsigned)((((uint64_t)a.n << a.lg) + THREADS - 1) / THREADS);
  if constexpr (WRITE) cache_write_kernel<T, VB, BITS, U><<<grid, THREADS, 0, s>>>(a, (const T*)rows);
  else cache_read_kernel<T, VB, BITS, U><<<grid, THREADS, 0, s>>>(a, (T*)rows);
}
template <bool WRITE, typename T, int VB, int BITS>
void launch_rows(const Move& a, void* rows, cudaStream_t s) {
  if (a.c.heads == 1) launch_heads<WRITE, T, VB, BITS, 1>(a, rows, s);
  else launch_heads<WRITE, T, VB, BITS, 2>(a, rows, s);
}
template <typename T, int VB, int BITS>
void launch_read_narrow(const Move& a, void* rows, cudaStream_t s) {
  const uint64_t lanes = ((uint64_t)a.n * a.c.heads) << (a.lg + 1);
  cache_read_narrow_kernel<T, VB, BITS><<<(unsigned)((lanes + THREADS - 1) / THREADS), THREADS, 0, s>>>(a, (T*)rows);
}

// Rows move in words of 16 bytes where base, row stride and head all start on one, else of 8, 4 or 2.  They are read by way of shared memory where
// that is a single value, and for pairs in fp32 of heads up to 64 wide, and always written straight from their words.
// 250 000 rows, straight and by shared memory, us.  Read from 4 bits: 8 x 25 in fp32 265 and 105, 8 x 43 347 and 199, 8 x 50 224 and 169,
// 8 x 43 in bf16 382 and 200, but 4 x 86 in fp32 164 and 164, 8 x 50 in bf16 139 and 169.  Written: 8 x 25 in fp32 118 and 119, 8 x 43 149 and 234, 8 x 50 103
// and 192, 8 x 43 in bf16 128 and 240.
template <bool WRITE, typename T, int BITS>
void launch_aligned(const Move& a, void* rows, cudaStream_t s) {
  constexpr int ES = (int)sizeof(T);
  const uint64_t at = (uint64_t)(uintptr_t)rows | (uint64_t)a.row_bytes | (uint64_t)(a.c.dim * ES);
  if ((at & 15) == 0) {
    launch_rows<WRITE, T, 16, BITS>(a, rows, s);
  } else if ((at & 7) == 0) {
    if constexpr (!WRITE && ES == 4) {
      if (a.c.dim <= 64) return launch_read_narrow<T, 8, BITS>(a, rows, s);
    }
    launch_rows<WRITE, T, 8, BITS>(a, rows, s);
  } else if (ES == 2 && (at & 3) == 0) {
    if constexpr (ES == 2) launch_rows<WRITE, T, 4, BITS>(a, rows, s);
  } else if constexpr (WRITE) {
    launch_rows<WRITE, T, ES, BITS>(a, rows, s);
  } else {
    launch_read_narrow<T, ES, BITS>(a, rows, s);
  }
}

template <bool WRITE>
int run(const char* who, const tgnn_cache* cache, void* rows, int dtype, int64_t num_rows, int64_t row_stride, const void* src,
        const void* dst, int index_bits, int64_t n, double* times, int32_t* status, void* stream, char* err, int64_t size) {
  Move a = {};
  const int rc = check_cache(who, "cache", cache, &a.c, err, size);
  if (rc) return rc;
  if (!known_dtype(dtype)) return fail(err, size, TGNN_EINVAL, "%s: unknown row type %d", who, dtype);
  if ((src || dst) && index_bits != 32 && index_bits != 64)
    return fail(err, size, TGNN_EINVAL, "%s: indices have 32 or 64 bits, not %d", who, index_bits);
  if (num_rows < 0 || n < 0 || row_stride < (int64_t)a.c.heads * a.c.dim)
    return fail(err, size, TGNN_EINVAL, "%s: size out of range (a row holds heads * dim values)", who);
  if (n > 0x7fffffff / a.c.heads) return fail(err, size, TGNN_ECAPACITY, "%s: n * heads beyond int32", who);
  if (num_rows > 0xffffffffll || a.c.rows > 0xffffffffll || row_stride > 0x7fffffff / elem_bytes(dtype))
    return fail(err, size, TGNN_ECAPACITY, "%s: 2^32 rows and more, or a row stride of 2^31 bytes and more", who);
  if (!status || (n > 0 && num_rows > 0 && !rows)) return fail(err, size, TGNN_EINVAL, "%s: null pointer", who);
  if (times && n > 0 && !a.c.times) return fail(err, size, TGNN_EINVAL, "%s: times given, but the cache holds none", who);
  const int idx = index_bits == 64 ? 7 : 3;
  if (((uintptr_t)rows & (elem_bytes(dtype) - 1)) || (((uintptr_t)src | (uintptr_t)dst) & idx) || ((uintptr_t)times & 7) ||
      ((uintptr_t)status & 3))
    return fail(err, size, TGNN_EINVAL, "%s: a pointer is not aligned to its element", who);
  if (n == 0) return TGNN_OK;
  a.num_rows = num_rows;
  a.row_bytes = (uint32_t)(row_stride * elem_bytes(dtype));
  a.src = src;
  a.dst = dst;
  a.index64 = index_bits == 64;
  a.n = (uint32_t)n;
  a.times = times;
  a.status = status;
  const int pad = padded_dim(a.c.dim);
  a.lg = pad == 32 ? 1 : pad == 64 ? 2 : 3;
  const bool four = a.c.bits == 4;
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == TGNN_F32) four ? launch_aligned<WRITE, float, 4>(a, rows, s) : launch_aligned<WRITE, float, 8>(a, rows, s);
  else if (dtype == TGNN_BF16) four ? launch_aligned<WRITE, __nv_bfloat16, 4>(a, rows, s) : launch_aligned<WRITE, __nv_bfloat16, 8>(a, rows, s);
  else four ? launch_aligned<WRITE, __half, 4>(a, rows, s) : launch_aligned<WRITE, __half, 8>(a, rows, s);
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
