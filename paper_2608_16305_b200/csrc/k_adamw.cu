// One AdamW step over many tensors in one launch, with moments in 32 or 8 bits.
//
//   g = grad * grad_scale;  m' = b1 m + (1 - b1) g;  v' = b2 v + ((1 - b2) g) g
//   p' = p - lr (decay p + (m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps))
//
// In 8 bits a block of 256 values has one scale each for m and for u = sqrt(v), and a value is c^2 * scale: codes that are squares
// resolve 16129 (m) and 65025 (u) to 1 within a block.  A value becomes one of its two neighbours by chance, so that the mean is right:
// a second moment that decays by 0.1 % a step would stay on its code for ever if it were rounded to the nearest.  u keeps code 1 where it is not 0, so
// that no step divides by eps alone.  Every operation up to the codes is one rounded fp32 operation (no contraction): codes are
// the same on every implementation.
//
// A warp takes 256 values at a time, eight per lane as two groups of four, which are 16-byte words of fp32 and 4-byte words of codes.
// Tensors are described in the kernel's parameters: nothing is copied to the device ahead of the launch, and a captured graph
// keeps them.  Bound by bytes: 28 per value with fp32 gradients and moments, 16 with moments in 8 bits.
#include <type_traits>

#include "tgnn_table.cuh"

using namespace tgnn_table;

namespace {

constexpr int kBlock = 256;                   // values per scale
constexpr int kThreads = 256;
constexpr float kLeast = 8.6736174e-19f;      // 2^-60: a block below it holds zeros

struct One {
  float* p;
  const void* g;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  void* copy;
  int64_t n;
  float decay;
  int8_t g_dtype, copy_dtype, wide;           // wide: every address is a multiple of four values
};
template <int MAX>
struct Many {
  One t[MAX];
  uint32_t end[MAX];                          // chunks up to and with tensor i
  int64_t* steps;                             // {steps done, blocks of this step that have read it}
  uint64_t seed;
  int64_t first;                              // place of t[0] in the caller's list
  double b1, b2, eps;
  float lr, grad_scale, b1f, b2f, n1, n2;
  uint32_t blocks;                            // of the launch that ends the step; 0: a later one does
  int count;
  int per_chunk;                              // values per thread block, a multiple of 2048
};

__device__ __forceinline__ uint64_t mix(uint64_t z) {  // SplitMix64's finaliser
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

// 1 - b^t in fp64 by squaring.
__device__ __forceinline__ double one_minus_power(double b, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return 1.0 - r;
}

// Four values (codes) from place `at` of a thread block's n on: words where `whole` says that all of them are there and aligned.
template <typename T>
__device__ __forceinline__ void load4(const T* p, int at, int n, bool whole, float* x) {
  if (whole) {
    reinterpret_cast<const Group<T, 4>*>(p + at)->get(x);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = at + i < n ? tgnn_history::to_float<T>(p[at + i]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, int at, int n, bool whole, const float* x) {
  if (whole) {
    Group<T, 4> g;
    g.set(x);
    *reinterpret_cast<Group<T, 4>*>(p + at) = g;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + i < n) p[at + i] = tgnn_history::from_float<T>(x[i]);
  }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int at, int n, bool whole) {
  if (whole) return *reinterpret_cast<const uint32_t*>(p + at);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (at + i < n) w |= (uint32_t)p[at + i] << (8 * i);
  return w;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int at, int n, bool whole, uint32_t w) {
  if (whole) *reinterpret_cast<uint32_t*>(p + at) = w;
  else
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + i < n) p[at + i] = (uint8_t)(w >> (8 * i));
}
// Conversions by bits: a byte under the exponent of 2^23 is a number behind it, and a sum with 2^23 (1.5 * 2^23 for signs) has its integer in the low
// bits.  The conversion instructions share the 16 lanes a cycle of the special functions: 8 of them per value would take longer than the memory.
__device__ __forceinline__ float byte_of(uint32_t w, int i) { return __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440u | i)); }   // + 2^23
__device__ __forceinline__ float signed_square(uint32_t codes_plus_128, int i, float scale) {
  const float c = byte_of(codes_plus_128, i) - 8388736.f;
  return __fmul_rn(c * fabsf(c), scale);      // squares up to 16129 are exact
}
__device__ __forceinline__ float square(uint32_t codes, int i, float scale) {
  const float c = byte_of(codes, i) - 8388608.f;
  return __fmul_rn(c * c, scale);
}
// Low bytes of four numbers.
__device__ __forceinline__ uint32_t low_bytes(const float* x) {
  const uint32_t a = __byte_perm(__float_as_uint(x[0]), __float_as_uint(x[1]), 0x0040), b = __byte_perm(__float_as_uint(x[2]), __float_as_uint(x[3]), 0x0040);
  return __byte_perm(a, b, 0x5410);
}

// Scale of a block whose largest magnitude (as bits, so that NaN stays on top) is `top`, and its reciprocal.
__device__ __forceinline__ float scale_of(uint32_t top_bits, float per, float* back) {
  const float top = __uint_as_float(top_bits);
  *back = 0.f;
  if (top_bits >= 0x7f800000u) return __uint_as_float(0x7fc00000u);           // reads back as NaN, all of it
  if (top < kLeast) return 0.f;
  const float s = __fmul_rn(top, per);
  *back = __frcp_rn(s);
  return s;
}
// The code of magnitude |x|: floor of the root, and one more by chance a in (0, 1).
__device__ __forceinline__ float code_of(float x, float back, float a, float most) {
  const float y = __fmul_rn(fabsf(x), back);
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  float c = (r + 8388608.f) - 8388608.f;      // the nearest integer: the root's floor or one more (the root is off by 2^-23 of it at most)
  if (c * c > y) c -= 1.f;                    // squares are exact
  if (y - c * c > __fmul_rn(a, 2.f * c + 1.f)) c += 1.f;                       // the difference is exact too
  return fminf(c, most);
}
__device__ __forceinline__ uint32_t warp_max(uint32_t x) { return __reduce_max_sync(FULL, x); }
// (h + 0.5) / 65536 of the low or the high 16 bits: 1 + h / 65536 by bits, less 1 - 2^-17; exact.
__device__ __forceinline__ float chance_low(uint32_t w) { return __uint_as_float(0x3f800000u | ((w << 7) & 0x7fff80u)) - 0.99999237060546875f; }
__device__ __forceinline__ float chance_high(uint32_t w) { return __uint_as_float(0x3f800000u | ((w >> 9) & 0x7fff80u)) - 0.99999237060546875f; }

template <int BITS, int MAX>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Many<MAX> a) {
  __shared__ float s_c1, s_c2;
  __shared__ uint64_t s_salt;
  if (threadIdx.x == 0) {
    volatile int64_t* const steps = a.steps;
    const int64_t t = steps[0] + 1;
    // The last block to have read the counter advances it: the others do not look at it again.  What a block announces is made of what it read (1 for any
    // number of steps), and what the last one writes of what it was told: a value cannot be its own cause, so no block reads the new one.
    unsigned long long before = 0;
    if (a.blocks > 0)
      asm volatile("{\n\t.reg .u64 one;\n\tshr.u64 one, %2, 63;\n\tadd.u64 one, one, 1;\n\tatom.add.gpu.global.u64 %0, [%1], one;\n\t}"
                   : "=l"(before)
                   : "l"(a.steps + 1), "l"(t)
                   : "memory");
    s_c1 = (float)(1.0 / one_minus_power(a.b1, t));
    s_c2 = (float)rsqrt(one_minus_power(a.b2, t));
    s_salt = a.seed ^ ((uint64_t)t * 0x9E3779B97F4A7C15ull);
    if (a.blocks > 0 && before == a.blocks - 1) {
      steps[0] = t;
      steps[1] = 0;
    }
  }
  int lo = 0, hi = a.count - 1;               // the tensor of this chunk: the first whose chunks end behind it
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.end[mid] > blockIdx.x) hi = mid;
    else lo = mid + 1;
  }
  const One& o = a.t[lo];
  const int64_t begin = (int64_t)(blockIdx.x - (lo ? a.end[lo - 1] : 0)) * a.per_chunk;
  const int n = (int)min(o.n - begin, (int64_t)a.per_chunk);        // of this block, from `begin` on
  const bool wide = o.wide;
  float* const op = o.p + begin;
  const int g_size = o.g_dtype == TGNN_F32 ? 4 : 2, state_size = BITS / 8;
  const char* const og = static_cast<const char*>(o.g) + begin * g_size;
  char *const om = static_cast<char*>(o.m) + begin * state_size, *const ov = static_cast<char*>(o.v) + begin * state_size;
  char* const oc = o.copy ? static_cast<char*>(o.copy) + begin * 2 : nullptr;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __syncthreads();
  const float c1 = s_c1, c2 = s_c2, eps = (float)a.eps;
  const uint64_t salt = s_salt;
  auto values = [&](const int at0, auto whole_) {
    constexpr bool whole = decltype(whole_)::value;
    float p[8], g[8], m[8], v[8];
    const int at[2] = {at0 + 4 * lane, at0 + 128 + 4 * lane};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      load4(op, at[h], n, whole, p + 4 * h);
      if (o.g_dtype == TGNN_F32) load4(reinterpret_cast<const float*>(og), at[h], n, whole, g + 4 * h);
      else if (o.g_dtype == TGNN_BF16) load4(reinterpret_cast<const __nv_bfloat16*>(og), at[h], n, whole, g + 4 * h);
      else load4(reinterpret_cast<const __half*>(og), at[h], n, whole, g + 4 * h);
    }
    const int64_t block = (begin + at0) / kBlock;
    if (BITS == 8) {
      uint32_t wm[2], wv[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        wm[h] = load_codes(reinterpret_cast<const uint8_t*>(om), at[h], n, whole);
        wv[h] = load_codes(reinterpret_cast<const uint8_t*>(ov), at[h], n, whole);
      }
      const float sm = o.m_scale[block], sv = o.v_scale[block];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        m[i] = signed_square(wm[i >> 2] ^ 0x80808080u, i & 3, sm);
        const float u = square(wv[i >> 2], i & 3, sv);
        v[i] = __fmul_rn(u, u);
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        load4(reinterpret_cast<const float*>(om), at[h], n, whole, m + 4 * h);
        load4(reinterpret_cast<const float*>(ov), at[h], n, whole, v + 4 * h);
      }
    }
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = __fmul_rn(g[i], a.grad_scale);
      m[i] = __fadd_rn(__fmul_rn(m[i], a.b1f), __fmul_rn(x, a.n1));
      v[i] = __fadd_rn(__fmul_rn(v[i], a.b2f), __fmul_rn(__fmul_rn(x, a.n2), x));
      u[i] = __fsqrt_rn(v[i]);
      // 1 - lr decay would round to fp32: the change is formed and taken off instead
      p[i] -= a.lr * fmaf(o.decay, p[i], m[i] * c1 * tgnn_history::rcp_fast(fmaf(u[i], c2, eps)));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      store4(op, at[h], n, whole, p + 4 * h);
      if (oc) {
        if (o.copy_dtype == TGNN_BF16) store4(reinterpret_cast<__nv_bfloat16*>(oc), at[h], n, whole, p + 4 * h);
        else store4(reinterpret_cast<__half*>(oc), at[h], n, whole, p + 4 * h);
      }
    }
    if (BITS == 8) {
      uint32_t tm = 0, tu = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {           // places behind the end were read as zeros and are zeros still
        tm = max(tm, __float_as_uint(m[i]) & 0x7fffffffu);
        tu = max(tu, __float_as_uint(u[i]) & 0x7fffffffu);
      }
      float bm, bu;
      const float sm = scale_of(warp_max(tm), 1.f / 16129.f, &bm), su = scale_of(warp_max(tu), 1.f / 65025.f, &bu);
      if (lane == 0) {
        o.m_scale[block] = sm;
        o.v_scale[block] = su;
      }
      constexpr uint64_t kPair = 0xC2B2AE3D27D4EB4Full;
      const uint64_t pair = (((uint64_t)(a.first + lo) << 40) + (uint64_t)((begin + at[0]) >> 1)) * kPair;     // those that follow are sums
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float cm[4], cu[4];
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const uint64_t r = mix(salt ^ (pair + (uint64_t)(64 * h + j / 2) * kPair));
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int i = 4 * h + j + e;
            const uint32_t w = (uint32_t)(r >> (32 * e));
            cm[j + e] = copysignf(code_of(m[i], bm, chance_low(w), 127.f), m[i]) + 12582912.f;
            float c = code_of(u[i], bu, chance_high(w), 255.f);
            if (c == 0.f && u[i] > 0.f && bu > 0.f) c = 1.f;
            cu[j + e] = c + 8388608.f;
          }
        }
        const uint32_t wm = low_bytes(cm), wv = low_bytes(cu);
        store_codes(reinterpret_cast<uint8_t*>(om), at[h], n, whole, wm);
        store_codes(reinterpret_cast<uint8_t*>(ov), at[h], n, whole, wv);
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        store4(reinterpret_cast<float*>(om), at[h], n, whole, m + 4 * h);
        store4(reinterpret_cast<float*>(ov), at[h], n, whole, v + 4 * h);
      }
    }
  };
  for (int at0 = warp * kBlock; at0 < n; at0 += (kThreads / 32) * kBlock) {
    if (wide && at0 + kBlock <= n) values(at0, std::true_type());
    else values(at0, std::false_type());
  }
}

// Moments in 8 bits as values: m into p's place of the description, v into copy's.
template <int MAX>
__global__ void __launch_bounds__(kThreads) moments_kernel(const __grid_constant__ Many<MAX> a) {
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.end[mid] > blockIdx.x) hi = mid;
    else lo = mid + 1;
  }
  const One& o = a.t[lo];
  const int64_t begin = (int64_t)(blockIdx.x - (lo ? a.end[lo - 1] : 0)) * a.per_chunk;
  const int n = (int)min(o.n - begin, (int64_t)a.per_chunk);
  const uint8_t *om = static_cast<const uint8_t*>(o.m) + begin, *ov = static_cast<const uint8_t*>(o.v) + begin;
  for (int at = 4 * threadIdx.x; at < n; at += 4 * kThreads) {
    const bool whole = o.wide && at + 4 <= n;
    const uint32_t wm = load_codes(om, at, n, whole), wv = load_codes(ov, at, n, whole);
    const int64_t block = (begin + at) / kBlock;
    const float sm = o.m_scale[block], sv = o.v_scale[block];
    float m[4], v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = signed_square(wm ^ 0x80808080u, i, sm);
      const float u = square(wv, i, sv);
      v[i] = __fmul_rn(u, u);
    }
    store4(o.p + begin, at, n, whole, m);
    store4(static_cast<float*>(o.copy) + begin, at, n, whole, v);
  }
}

// Values per thread block: 2048, so that few values have many blocks.  With moments in 8 bits, where a block's set-up (the powers of b1 and b2) is felt
// beside its arithmetic, 8192 where enough blocks remain (us with 2048 / 8192 / 16384: 4M values 21 / 22 / 24, 10M 49 / 47 / 52, 20M 93 / 92 / 89,
// 60M 269 / 248 / 233, 26M in 18 tensors - / 173 / 184; with moments in 32 bits 2048 is best throughout: 10M 44 / 48 / 52, 60M 244 / 251 / 258).
int per_chunk_of(int64_t values, int bits) { return bits == 8 && values / (8 * num_sms()) >= 8192 ? 8192 : 2048; }

template <int MAX, typename K>
void launch(K kernel, Chain& c, const tgnn_adamw_tensor* t, float* const* m_out, float* const* v_out, int from, int count, int bits, Many<MAX>& a,
            bool ends, int per_chunk) {
  uint64_t chunks = 0;
  a.first = from;
  a.count = count;
  a.per_chunk = per_chunk;
  for (int i = 0; i < count; ++i) {
    const tgnn_adamw_tensor& x = t[from + i];
    One& o = a.t[i];
    o.p = m_out ? m_out[from + i] : x.param;
    o.g = x.grad;
    o.m = x.m;
    o.v = x.v;
    o.m_scale = x.m_scale;
    o.v_scale = x.v_scale;
    o.copy = v_out ? v_out[from + i] : x.copy;
    o.n = x.numel;
    o.decay = x.weight_decay;
    o.g_dtype = (int8_t)x.grad_dtype;
    o.copy_dtype = (int8_t)x.copy_dtype;
    const uintptr_t mv = (uintptr_t)x.m | (uintptr_t)x.v;
    o.wide = ((uintptr_t)o.p & 15) == 0 && (mv & (bits == 8 ? 3 : 15)) == 0 && ((uintptr_t)o.copy & (v_out ? 15 : 7)) == 0 &&
             (m_out || ((uintptr_t)x.grad & (4 * elem_bytes(x.grad_dtype) - 1)) == 0);
    chunks += (uint64_t)((x.numel + per_chunk - 1) / per_chunk);
    a.end[i] = (uint32_t)chunks;
  }
  a.blocks = ends ? (uint32_t)chunks : 0;
  if (chunks) c(kernel, dim3((unsigned)chunks), dim3(kThreads), 0, a);
}

int check(const char* who, const tgnn_adamw_tensor* t, int count, int bits, bool read, int64_t* values, int* used, char* err, int64_t size) {
  if (bits != 8 && bits != 32) return fail(err, size, TGNN_EINVAL, "%s: state_bits is 8 or 32", who);
  if (count < 0 || (count > 0 && !t)) return fail(err, size, TGNN_EINVAL, "%s: no tensors given", who);
  if (count > 1 << 20) return fail(err, size, TGNN_ECAPACITY, "%s: more than 2^20 tensors", who);
  *values = 0;
  *used = 0;
  for (int i = 0; i < count; ++i) {
    const tgnn_adamw_tensor& x = t[i];
    if (x.numel < 0 || x.numel > 1ll << 40) return fail(err, size, TGNN_EINVAL, "%s: tensor %d: size out of range", who, i);
    if (x.numel == 0) continue;
    if (!x.m || !x.v || (bits == 8 && (!x.m_scale || !x.v_scale)) || (!read && (!x.param || !x.grad)))
      return fail(err, size, TGNN_EINVAL, "%s: tensor %d: null pointer", who, i);
    if (!read && (!known_dtype(x.grad_dtype) || (x.copy && x.copy_dtype != TGNN_BF16 && x.copy_dtype != TGNN_F16)))
      return fail(err, size, TGNN_EINVAL, "%s: tensor %d: a gradient is fp32, bf16 or fp16, a copy bf16 or fp16", who, i);
    if (((uintptr_t)x.param & 3) || ((bits == 32) && (((uintptr_t)x.m | (uintptr_t)x.v) & 3)) || (((uintptr_t)x.m_scale | (uintptr_t)x.v_scale) & 3) ||
        ((uintptr_t)x.copy & 1) || (!read && ((uintptr_t)x.grad & (elem_bytes(x.grad_dtype) - 1))))
      return fail(err, size, TGNN_EINVAL, "%s: tensor %d: a pointer is not aligned to its element", who, i);
    *values += x.numel;
    *used = i + 1;
  }
  if (*values > 1ll << 42) return fail(err, size, TGNN_ECAPACITY, "%s: more than 2^42 values", who);
  return TGNN_OK;
}

constexpr int kFew = 40, kMost = 360;          // tensors of one launch: 4 KB of parameters, or 32 KB

}  // namespace

extern "C" TGNN_API int64_t tgnn_adamw_blocks(int64_t numel) { return numel < 0 ? -1 : (numel + kBlock - 1) / kBlock; }

extern "C" TGNN_API int tgnn_adamw_step(const tgnn_adamw_tensor* tensors_host, int count, int state_bits, int64_t* steps, double lr, double beta1,
                                        double beta2, double eps, double grad_scale, uint64_t seed, void* stream, char* err, int64_t err_size) {
  const char* who = "tgnn_adamw_step";
  int64_t values;
  int used;
  if (int rc = check(who, tensors_host, count, state_bits, false, &values, &used, err, err_size)) return rc;
  const float b1 = (float)beta1, b2 = (float)beta2;
  if (!(lr >= 0) || !(beta1 >= 0 && b1 < 1.f) || !(beta2 >= 0 && b2 < 1.f) || !(eps >= 0) || !(grad_scale - grad_scale == 0))
    return fail(err, err_size, TGNN_EINVAL, "%s: lr >= 0, 0 <= beta < 1 (in fp32, too), eps >= 0 and a finite grad_scale are needed", who);
  if (eps > 0 && !((float)eps >= 1.17549435e-38f))         // the quotient's reciprocal takes what is smaller for 0: a value without gradients would be 0 / 0
    return fail(err, err_size, TGNN_EINVAL, "%s: eps is below the smallest normal number of fp32 and not 0", who);
  if (!steps || ((uintptr_t)steps & 7)) return fail(err, err_size, TGNN_EINVAL, "%s: steps is null or not 8-byte aligned", who);
  if (values == 0) return TGNN_OK;
  const int per = per_chunk_of(values, state_bits);
  Chain c(stream);
  auto fill = [&](auto& a) {
    a.steps = steps;
    a.seed = seed;
    a.b1 = b1;                                 // one number in the moments and in their corrections: with 0.9999 in fp64 there, 1 - beta would be 1.7e-4 off
    a.b2 = b2;
    a.eps = eps;
    a.lr = (float)lr;
    a.grad_scale = (float)grad_scale;
    a.b1f = b1;
    a.b2f = b2;
    a.n1 = 1.f - b1;                           // exact from 0.5 on
    a.n2 = 1.f - b2;
  };
  for (int from = 0; from < used;) {
    c.first = true;                            // launches of one step touch different tensors, and the counter in stream order
    if (used - from <= kFew) {
      Many<kFew> a;
      fill(a);
      launch(state_bits == 8 ? adamw_kernel<8, kFew> : adamw_kernel<32, kFew>, c, tensors_host, nullptr, nullptr, from, used - from, state_bits, a, true,
             per);
      from = used;
    } else {
      Many<kMost> a;
      fill(a);
      const int now = used - from < kMost ? used - from : kMost;
      launch(state_bits == 8 ? adamw_kernel<8, kMost> : adamw_kernel<32, kMost>, c, tensors_host, nullptr, nullptr, from, now, state_bits, a,
             from + now == used, per);
      from += now;
    }
  }
  return c.end(who, err, err_size);
}

extern "C" TGNN_API int tgnn_adamw_moments(const tgnn_adamw_tensor* tensors_host, int count, float* const* m_out_host, float* const* v_out_host,
                                           void* stream, char* err, int64_t err_size) {
  const char* who = "tgnn_adamw_moments";
  int64_t values;
  int used;
  if (int rc = check(who, tensors_host, count, 8, true, &values, &used, err, err_size)) return rc;
  if (values == 0) return TGNN_OK;
  if (!m_out_host || !v_out_host) return fail(err, err_size, TGNN_EINVAL, "%s: null pointer", who);
  for (int i = 0; i < used; ++i)
    if (tensors_host[i].numel > 0 && (!m_out_host[i] || !v_out_host[i] || (((uintptr_t)m_out_host[i] | (uintptr_t)v_out_host[i]) & 3)))
      return fail(err, err_size, TGNN_EINVAL, "%s: tensor %d: an output is null or not aligned", who, i);
  const int per = per_chunk_of(values, 8);
  Chain c(stream);
  for (int from = 0; from < used;) {
    c.first = true;
    const int most = used - from <= kFew ? kFew : kMost, now = used - from < most ? used - from : most;
    if (most == kFew) {
      Many<kFew> a = {};
      launch(moments_kernel<kFew>, c, tensors_host, m_out_host, v_out_host, from, now, 8, a, false, per);
    } else {
      Many<kMost> a = {};
      launch(moments_kernel<kMost>, c, tensors_host, m_out_host, v_out_host, from, now, 8, a, false, per);
    }
    from += now;
  }
  return c.end(who, err, err_size);
}
