// Attention of one query per root and head over the window and the sinks of the root's history, keys and values in a row cache
// of 4 or 8 bits, with a learned bias by buckets of the time difference.
//
//   s_j = scale * q . k_j + bias[h, bucket_j],   k_j = ks_j * c_j   (c_j: integer codes, one scale per row and head)
//   out = sum_j p_j v_j / l,   p_j = exp(s_j - m),  l = sum_j p_j    (m = running maximum)
// (Logits stay in natural units, and log2(e) goes into the difference: a bias of the type's lowest value is then still finite.)
//
// Both products run on the tensor cores (m16n8k16, fp16 operands, fp32 sums) although a root has a single query: what they save is not
// the multiplications but the conversion of every code to fp32 and the sums across lanes.  Codes are the 16-row operand (16 keys,
// or 16 columns of the values), queries and weights the 8 columns: two for each of four query heads that share a cached head.
// Those two hold a number x as hi + lo / 2048 in fp16 (22 bits), and both products of a head end up in one thread.  (Weights below 2^-14 of the
// largest have fewer, those below 2^-36 of it are lost: less than fp32's sums lose beside the largest.)
// Codes go in as fp16 integers (exact), centred: their bits under the exponent of 1024 minus 1024 and the stored offset.  (Under a zero
// exponent a mask alone would unpack them, but the tensor core lines products up by their nominal exponents, and sums of such
// numbers came out at 2^-17.)  Scales are applied to the other side: ks_j to the finished logits, vs_j to the weights.  fp16's range is
// no limit: a query is divided by a power of two at its largest value, and weights w_j = p_j vs_j are divided by a running bound
// sc of w.  The output is held in units of sc at maximum m;
// when a weight passes sc it is rescaled.
//
// The sum over dim may be taken in any order, so a lane reads neighbouring words of a key's codes with one wide load and the query
// is laid out to match; likewise for the values' columns.  tcgen05's tiles have 128 rows that share one operand; here every root
// brings rows of its own, 20 to a few hundred, and each with its own mask.
//
// Work: a unit is a root, a cached head and up to 4 of its query heads (8 where more share it).  Units are handled by a warp, by a block of 4 warps
// or by a cluster of 2 to 16 blocks whose partial results meet in distributed shared memory (no workspace, no atomics, sums in
// a fixed order); the launch takes more warps per unit while the units alone would leave SMs idle and each warp still has a few
// tiles to walk.
//
// Measured on a B200: 12 000 roots over 520 entries, 8 heads over 2 cached ones of 64, 4 bits: 206 us, 1.6 TB/s of DRAM traffic (neighbouring
// roots share rows in L2) and 33 TFLOP/s; 1800 roots over 66 entries, 2 heads of 50, 8 bits: 14.5 us; 14 400 over 21, 4 bits: 39 us; three roots
// over 4100 entries: 7.5 us.  What bounds it is instructions, 2.3 per cycle and SM from 20 warps (24 with registers to spare fetch no more,
// 16 take 16 % longer): a tile of 32 keys of 64 costs 545, of which unpacking takes 152 and the products 16; the rest is softmax, bias,
// addresses and loads.  The
// smallest calls are bound by the chain of dependent loads (length, rows, then the sums' meeting).
#include <cooperative_groups.h>

#include "attend_shape.h"
#include "tgnn_history.cuh"

using namespace tgnn_history;
namespace cg = cooperative_groups;

namespace {

constexpr int WARPS = kAttendWarps;
constexpr float kLo = 2048.f;             // lo terms are held times 2^11, clear of fp16's subnormals

struct AttendArgs {
  const void* q;
  void* out;
  int dtype;
  const uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
  uint32_t k_code_stride, v_code_stride, k_scale_stride, v_scale_stride;
  int64_t rows;
  uint32_t units;
  int heads, kv_heads, group, passes, dim;    // group = heads / kv_heads, passes = ceil(group / heads of a unit)
  int take;                                   // units of a warp: 1, or all of a root (passes * kv_heads)
  const int64_t* first;
  const int32_t* len;
  const float* bias;
  const double *bounds, *times, *ts;
  int buckets, window, sinks;
  float scale;
  int32_t* status;
  bool pairs;                                 // q and out may be read and written two values at a time
};

__device__ const float no_bias = 0.f;         // read where there is no bias (buckets = 0: by every head)

__device__ __forceinline__ uint32_t h2u(__half2 x) { return *reinterpret_cast<uint32_t*>(&x); }
__device__ __forceinline__ __half2 u2h(uint32_t x) { return *reinterpret_cast<__half2*>(&x); }

// (a & mask) | bits
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t mask, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(a), "r"(mask), "r"(bits));
  return r;
}

// The four pairs of codes whose nibbles lie in the low and the high half of t: out[j] = (nibble j, nibble j + 4) - 8 as fp16.  A nibble
// under the exponent of 1024 reads as 1024 + n, four bits further up as 1024 + 16 n.
__device__ __forceinline__ void nibbles(uint32_t t, uint32_t (&out)[4]) {
  const __half2 one = u2h(0x64086408u);                                 // 1032
  const __half2 sixteenth = u2h(0x2c002c00u), off = u2h(0xd480d480u);   // 1 / 16, -72
  out[0] = h2u(__hsub2(u2h(and_or(t, 0x000f000fu, 0x64006400u)), one));
  out[1] = h2u(__hfma2(u2h(and_or(t, 0x00f000f0u, 0x64006400u)), sixteenth, off));
  t >>= 8;
  out[2] = h2u(__hsub2(u2h(and_or(t, 0x000f000fu, 0x64006400u)), one));
  out[3] = h2u(__hfma2(u2h(and_or(t, 0x00f000f0u, 0x64006400u)), sixteenth, off));
}
// Two bytes under the exponent of 1024, minus 1024 and their offset of 128.
__device__ __forceinline__ uint32_t centre(uint32_t x) { return h2u(__hsub2(u2h(x), u2h(0x64806480u))); }

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// x0, x1 as fp16 pairs hi and lo with x = hi + lo / 2048
__device__ __forceinline__ void split2(float x0, float x1, uint32_t* hi, uint32_t* lo) {
  const __half2 h = __floats2half2_rn(x0, x1);
  const float2 f = __half22float2(h);
  *hi = h2u(h);
  *lo = h2u(__floats2half2_rn((x0 - f.x) * kLo, (x1 - f.y) * kLo));
}

// N neighbouring words (or, for B = 2, a half word) from shared memory.
template <int B>
struct Piece { uint32_t w[(B + 3) / 4]; };
template <int B>
__device__ __forceinline__ Piece<B> load_piece(const uint8_t* p) {
  Piece<B> r;
  if constexpr (B == 2) {
    r.w[0] = *reinterpret_cast<const uint16_t*>(p);
  } else if constexpr (B == 4) {
    r.w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (B == 8) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    r.w[0] = x.x;
    r.w[1] = x.y;
  } else {
#pragma unroll
    for (int i = 0; i < B / 16; ++i) {
      const uint4 x = *(reinterpret_cast<const uint4*>(p) + i);
      r.w[4 * i] = x.x;
      r.w[4 * i + 1] = x.y;
      r.w[4 * i + 2] = x.z;
      r.w[4 * i + 3] = x.w;
    }
  }
  return r;
}

// N values of a query row from column e0 on, as fp32 (0 beyond dim): in pairs where every row starts on one.
template <int N>
__device__ __forceinline__ void load_query(const AttendArgs& a, int64_t base, int e0, bool on, float (&x)[N]) {
  if (a.pairs) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const bool in = on && e0 + i < a.dim;
      float2 f = make_float2(0.f, 0.f);
      if (a.dtype == TGNN_F32) {
        if (in) f = __ldg(reinterpret_cast<const float2*>(reinterpret_cast<const float*>(a.q) + base + e0 + i));
      } else {
        uint32_t w = 0;
        if (in) w = __ldg(reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint16_t*>(a.q) + base + e0 + i));
        if (a.dtype == TGNN_BF16) f = make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
        else f = __half22float2(u2h(w));
      }
      x[i] = f.x;
      x[i + 1] = f.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = 0.f;
      if (on && e0 + i < a.dim) {
        if (a.dtype == TGNN_F32) x[i] = __ldg(reinterpret_cast<const float*>(a.q) + base + e0 + i);
        else if (a.dtype == TGNN_BF16) x[i] = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(a.q)[base + e0 + i]);
        else x[i] = __half2float(reinterpret_cast<const __half*>(a.q)[base + e0 + i]);
      }
    }
  }
}
// (fp16: a mean of values that a cache holds at the type's end, which its rounded scale puts up to 2^-7 past it, stays finite.)
__device__ __forceinline__ void store_out(const AttendArgs& a, int64_t i, float x) {
  if (a.dtype == TGNN_F32) reinterpret_cast<float*>(a.out)[i] = x;
  else if (a.dtype == TGNN_BF16) reinterpret_cast<__nv_bfloat16*>(a.out)[i] = __float2bfloat16_rn(x);
  else reinterpret_cast<__half*>(a.out)[i] = __float2half_rn(within<__half>(x));
}
// Columns e and e + 1 of an output row: e is even, the row a pair's multiple long.
__device__ __forceinline__ void store_pair(const AttendArgs& a, int64_t i, float x, float y) {
  if (a.dtype == TGNN_F32) {
    *reinterpret_cast<float2*>(reinterpret_cast<float*>(a.out) + i) = make_float2(x, y);
  } else if (a.dtype == TGNN_BF16) {
    *reinterpret_cast<__nv_bfloat162*>(reinterpret_cast<__nv_bfloat16*>(a.out) + i) = __floats2bfloat162_rn(x, y);
  } else {
    *reinterpret_cast<__half2*>(reinterpret_cast<__half*>(a.out) + i) = __floats2half2_rn(within<__half>(x), within<__half>(y));
  }
}

// Keys that a warp takes at a time: 32, or 16 where 32 rows take 8 KB of shared memory.
template <int BITS, int DP>
struct Tile {
  static constexpr int TK = BITS * DP >= 1024 ? 16 : 32;
  static constexpr int NT = TK / 8;                 // keys whose logits a lane has: 8 j + lane / 4
  static constexpr int KW = DP * BITS / 128;        // words of a key that a lane reads (a quarter of the row)
  static constexpr int VD = DP / 8;                 // columns of a value that a lane reads
  static constexpr int VB = VD * BITS / 8;          // bytes of them: 2 to 16
  static constexpr int RB = DP * BITS / 8;          // bytes of a row's head
};

// A root's visible entries: u < ns are the sinks, the others lie `skip` further on.  The pointers are those of entry 0 for the lane's
// part of a row (codes, of the unit's cached head) and for whole rows (scales of that head, times).
struct Seen {
  int n, ns, skip;
  double t;
  const uint8_t *k, *v, *ks, *vs;
  const double* ts;
  __device__ __forceinline__ uint32_t entry(int u) const {          // beyond the last entry: the last (its weight is set to 0)
    u = min(u, n - 1);
    return (uint32_t)(u < ns ? u : u + skip);
  }
};

// One tile on its way: codes by asynchronous copies to the warp's shared memory (keys, then values, row by row), the scales and time of
// one key in registers: key `lane`, or for a single head the lane's own one (8 (lane % 4) + lane / 4).
template <int BITS, int DP, bool ONE>
struct Rows {
  using T = Tile<BITS, DP>;
  uint32_t scales;
  double ts;

  __device__ __forceinline__ void load(const AttendArgs& a, const Seen& seen, int tile, uint32_t to) {
    const int lane = threadIdx.x & 31, u0 = tile * T::TK;
    constexpr int CPR = T::RB / 16, PER = 32 / CPR;                 // 16-byte pieces of a row, rows per copy of the warp
#pragma unroll
    for (int i = 0; i < T::TK / PER; ++i) {
      const uint32_t e = seen.entry(u0 + i * PER + lane / CPR);
      const uint8_t *kp = seen.k + (uint64_t)e * a.k_code_stride, *vp = seen.v + (uint64_t)e * a.v_code_stride;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 512 * i), "l"(kp) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + T::TK * T::RB + 512 * i), "l"(vp) : "memory");
    }
    const int u = u0 + ((ONE ? 8 * (lane & 3) + (lane >> 2) : lane) & (T::TK - 1));
    const uint32_t e = seen.entry(u);
    const uint32_t ks = __ldg(reinterpret_cast<const uint16_t*>(seen.ks + (uint64_t)e * a.k_scale_stride));
    const uint32_t vs = __ldg(reinterpret_cast<const uint16_t*>(seen.vs + (uint64_t)e * a.v_scale_stride));
    scales = u < seen.n ? ks | vs << 16 : 0;                        // hidden keys' values weigh nothing
    if (a.bias) ts = __ldg(seen.ts + e);
  }
};

// The largest of a warp's values, NaN left out.
__device__ __forceinline__ float max_warp(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}

// A unit's running sums over the tiles that one warp walks, for 4 NH heads; NH = 0: for a single one, which then fills all columns, so
// that every lane has its logits and takes one key of the tile to itself (11 % less time than as one of four heads).
// Lane (g, c) has head c of every four: its logits at keys
// 16 b + g and 16 b + g + 8, its output columns g VD + i at o[i / 2][.][2 (i & 1) + {hi, lo}] in units of sc, its sum l over the
// lane's own keys until finish().
template <int BITS, int DP, int NH>
struct Walk {
  using T = Tile<BITS, DP>;
  static constexpr bool ONE = NH == 0;
  static constexpr int KS = DP / 16, MT = T::VD / 2, X = ONE ? 1 : NH;
  float o[MT][X][4];
  float m[X], l[X], sc[X], qfac[X];
  uint32_t qb[X][KS][2];

  __device__ __forceinline__ void none() {
#pragma unroll
    for (int x = 0; x < X; ++x) {
      m[x] = -INFINITY;
      l[x] = sc[x] = 0.f;
#pragma unroll
      for (int i = 0; i < MT; ++i) o[i][x][0] = o[i][x][1] = o[i][x][2] = o[i][x][3] = 0.f;
    }
  }

  // The query of a single head.  All eight lanes of a quarter need the same columns, so each prepares two or four of them and they meet
  // in shared memory (`to`: 4 DP bytes of the warp's own), in the order in which the lanes read them: hi terms, then lo terms.
  __device__ __forceinline__ void begin_one(const AttendArgs& a, int64_t root, int head, uint32_t* to) {
    none();
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    constexpr int PAIRS = DP / 64 > 0 ? DP / 64 : 1;                 // of columns per lane (DP 32: every other lane has one)
    float x[PAIRS][2], top = 0.f;
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
      const int e = c * (DP / 4) + 2 * (g * PAIRS + i);
      load_query<2>(a, (root * a.heads + head) * a.dim, e, DP >= 64 || g < 4, x[i]);
      top = fmaxf(top, fmaxf(fabsf(x[i][0]), fabsf(x[i][1])));
    }
    top = max_warp(top);
    // 2^e <= top < 2^(e + 1): scaled queries lie below 2 (infinities and NaN stay what they are)
    const int e = min(max((int)(__float_as_uint(top) >> 23), 2), 252);
    const float down = __uint_as_float((uint32_t)(254 - e) << 23);
    qfac[0] = a.scale * __uint_as_float((uint32_t)e << 23);
    __half* hi = reinterpret_cast<__half*>(to) + c * (DP / 4);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int d = 2 * (g * PAIRS + i) + k;                       // column of the quarter
        // its place: columns j and j + 4 of every 8 share a word where nibbles are paired so
        const int at = BITS == 4 ? (d & ~7) + 2 * (d & 3) + ((d >> 2) & 1) : d;
        const float y = x[i][k] * down;
        const __half h = __float2half_rn(y);
        if (DP >= 64 || g < 4) {
          hi[at] = h;
          hi[DP + at] = __float2half_rn((y - __half2float(h)) * kLo);
        }
      }
    }
    __syncwarp();
    const uint32_t* mine = to + (g & 1) * (DP / 2) + c * (DP / 8);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qb[0][s][0] = mine[2 * s];
      qb[0][s][1] = mine[2 * s + 1];
    }
    __syncwarp();                                                    // the next unit's query may be written
  }

  // The query of several heads: lane (g, c) holds columns [c DP / 4, (c + 1) DP / 4) of head g / 2 of every four, the hi terms where g is even, lo
  // where it is odd, divided by a power of two.
  __device__ __forceinline__ void begin(const AttendArgs& a, int64_t root, int head0, int nh) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    none();
#pragma unroll
    for (int x = 0; x < X; ++x) {
      const int h = 4 * x + (g >> 1);
      float q[DP / 4];
      load_query<DP / 4>(a, (root * a.heads + head0 + h) * a.dim, c * (DP / 4), h < nh, q);
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < DP / 4; ++i) top = fmaxf(top, fabsf(q[i]));
      top = fmaxf(top, __shfl_xor_sync(FULL, top, 1));
      top = fmaxf(top, __shfl_xor_sync(FULL, top, 2));
      // 2^e <= top < 2^(e + 1): scaled queries lie below 2 (infinities and NaN stay what they are)
      const int e = min(max((int)(__float_as_uint(top) >> 23), 2), 252);
      const float down = __uint_as_float((uint32_t)(254 - e) << 23);
      qfac[x] = a.scale * __uint_as_float((uint32_t)__shfl_sync(FULL, e, 8 * c) << 23);       // to the lanes of the head's logits
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        // BITS 4: the columns of a step in the order in which nibbles() pairs them
        const int b = BITS == 4 ? 8 * (s >> 1) + 2 * (s & 1) : 4 * s;
        const int i1 = BITS == 4 ? b + 4 : b + 1, i2 = BITS == 4 ? b + 1 : b + 2, i3 = BITS == 4 ? b + 5 : b + 3;
        uint32_t hi, lo;
        split2(q[b] * down, q[i1] * down, &hi, &lo);
        qb[x][s][0] = (g & 1) ? lo : hi;
        split2(q[i2] * down, q[i3] * down, &hi, &lo);
        qb[x][s][1] = (g & 1) ? lo : hi;
      }
    }
  }

  __device__ __forceinline__ void tile(const AttendArgs& a, const float* bias, const Seen& seen, uint32_t scales, int bucket, const uint8_t* rows,
                                       int u0, int nh) {
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    // logits: s[x][j] of head 4 x + c at key 8 j + g
    float s[X][T::NT];
#pragma unroll
    for (int b = 0; b < T::NT / 2; ++b) {
      float acc[X][4];
#pragma unroll
      for (int x = 0; x < X; ++x) acc[x][0] = acc[x][1] = acc[x][2] = acc[x][3] = 0.f;
      const auto r0 = load_piece<T::RB / 4>(rows + (16 * b + g) * T::RB + c * (T::RB / 4));
      const auto r1 = load_piece<T::RB / 4>(rows + (16 * b + 8 + g) * T::RB + c * (T::RB / 4));
#pragma unroll
      for (int w = 0; w < T::KW; ++w) {
        const uint32_t k0 = r0.w[w], k1 = r1.w[w];
        if constexpr (BITS == 4) {
          uint32_t p[4], q[4];
          nibbles(k0, p);
          nibbles(k1, q);
#pragma unroll
          for (int x = 0; x < X; ++x) {
            mma(acc[x], p[0], q[0], p[1], q[1], qb[x][2 * w][0], qb[x][2 * w][1]);
            mma(acc[x], p[2], q[2], p[3], q[3], qb[x][2 * w + 1][0], qb[x][2 * w + 1][1]);
          }
        } else {
          const uint32_t p0 = centre(__byte_perm(k0, 0x64646464u, 0x4140)), p1 = centre(__byte_perm(k0, 0x64646464u, 0x4342));
          const uint32_t q0 = centre(__byte_perm(k1, 0x64646464u, 0x4140)), q1 = centre(__byte_perm(k1, 0x64646464u, 0x4342));
#pragma unroll
          for (int x = 0; x < X; ++x) mma(acc[x], p0, q0, p1, q1, qb[x][w][0], qb[x][w][1]);
        }
      }
#pragma unroll
      for (int x = 0; x < X; ++x) {
        s[x][2 * b] = fmaf(acc[x][1], 1.f / kLo, acc[x][0]);
        s[x][2 * b + 1] = fmaf(acc[x][3], 1.f / kLo, acc[x][2]);
      }
    }
    uint32_t mine = 0;                                                // ONE: the weight of the lane's own key, hi and lo
    if constexpr (ONE) {
      const int j = c & (T::NT - 1), key = 8 * j + g;
      float z = s[0][0];
#pragma unroll
      for (int i = 1; i < T::NT; ++i) z = j == i ? s[0][i] : z;
      z = fmaf(z, qfac[0] * __uint_as_float(scales << 16), __ldg(bias + bucket));
      if (u0 + key >= seen.n) z = -INFINITY;
      const float top = fmaxf(m[0], max_warp(z));
      const float base = top == -INFINITY ? 0.f : top;               // nothing but -infinity so far: weights are 0
      const float corr = exp2_fast((m[0] - base) * kLog2e);          // m = -infinity: 0
      m[0] = top;
      const float p = exp2_fast((z - base) * kLog2e);
      l[0] = fmaf(l[0], corr, c < T::NT ? p : 0.f);                // 16 keys: lanes c >= 2 repeat the others'
      const float w = p * __uint_as_float(scales & 0xffff0000u), wmax = max_warp(w);
      const bool some = sc[0] != 0.f;                                // not the first tile: there are sums (corr may be 0)
      sc[0] *= corr;                                                 // a larger maximum shrinks the unit of the sums, not the sums
      const float need = __uint_as_float(min(max((__float_as_uint(wmax) >> 23) + 1u, 2u), 252u) << 23);   // 2^e > wmax
      const float old = sc[0];
      const bool grow = need > old;
      sc[0] = grow ? need : old;
      const float inv = rcp_fast(sc[0]);
      if (grow && some) {
        const float f = old * inv;
#pragma unroll
        for (int i = 0; i < MT; ++i) { o[i][0][0] *= f; o[i][0][1] *= f; o[i][0][2] *= f; o[i][0][3] *= f; }
      }
      const float ws = w * inv;
      const __half hi = __float2half_rn(ws);
      const __half lo = __float2half_rn((ws - __half2float(hi)) * kLo);
      mine = (uint32_t)__half_as_ushort(hi) | (uint32_t)__half_as_ushort(lo) << 16;
    } else {
      float vs[T::NT], top[X];
#pragma unroll
      for (int x = 0; x < X; ++x) top[x] = m[x];
#pragma unroll
      for (int j = 0; j < T::NT; ++j) {
        const int key = 8 * j + g;
        const uint32_t two = __shfl_sync(FULL, scales, key);
        const float ks = __uint_as_float(two << 16);
        vs[j] = __uint_as_float(two & 0xffff0000u);
        const int at = __shfl_sync(FULL, bucket, key);
#pragma unroll
        for (int x = 0; x < X; ++x) {
          const float z = fmaf(s[x][j], qfac[x] * ks, __ldg(bias + min(4 * x + c, nh - 1) * a.buckets + at));
          s[x][j] = u0 + key < seen.n ? z : -INFINITY;
          top[x] = fmaxf(top[x], s[x][j]);
        }
      }
      float wmax[X];
#pragma unroll
      for (int x = 0; x < X; ++x) {
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) top[x] = fmaxf(top[x], __shfl_xor_sync(FULL, top[x], w));
        const float base = top[x] == -INFINITY ? 0.f : top[x];         // nothing but -infinity so far: weights are 0
        const float corr = exp2_fast((m[x] - base) * kLog2e);          // m = -infinity: 0
        m[x] = top[x];
        float sum = 0.f;
        wmax[x] = 0.f;
#pragma unroll
        for (int j = 0; j < T::NT; ++j) {
          const float p = exp2_fast((s[x][j] - base) * kLog2e);
          sum += p;
          s[x][j] = p * vs[j];
          wmax[x] = fmaxf(wmax[x], s[x][j]);
        }
        l[x] = fmaf(l[x], corr, sum);
        const bool some = sc[x] != 0.f;                                // not the first tile: there are sums (corr may be 0)
        sc[x] *= corr;                                                 // a larger maximum shrinks the unit of the sums, not the sums
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) wmax[x] = fmaxf(wmax[x], __shfl_xor_sync(FULL, wmax[x], w));
        const float need = __uint_as_float(min(max((__float_as_uint(wmax[x]) >> 23) + 1u, 2u), 252u) << 23);   // 2^e > wmax
        const bool grow = need > sc[x];
        const float old = sc[x];
        sc[x] = grow ? need : old;
        const float inv = rcp_fast(sc[x]);
        if (__any_sync(FULL, grow && some)) {
          const float f = grow ? old * inv : 1.f;
#pragma unroll
          for (int i = 0; i < MT; ++i) { o[i][x][0] *= f; o[i][x][1] *= f; o[i][x][2] *= f; o[i][x][3] *= f; }
        }
#pragma unroll
        for (int j = 0; j < T::NT; ++j) s[x][j] *= inv;
      }
    }
    // output: 16 keys at a time, in the order c, c + 4, c + 8, c + 12 for lane (g, c), whose values' rows then lie in different banks.
    // The weights go from (key, head) lanes to (column, key) lanes: column g is head g / 2, hi or lo.
    const int from = 4 * c + (g >> 1);
    rows += T::TK * T::RB + g * T::VB + c * T::RB;
#pragma unroll
    for (int t = 0; t < T::TK / 16; ++t) {
      uint32_t pb[X][2];
      if constexpr (ONE) {
        const uint32_t sel = (g & 1) ? 0x7632 : 0x5410;              // hi or lo terms of two keys; key 8 i + k is lane 4 k + i's
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t ka = __shfl_sync(FULL, mine, 4 * c + 2 * t + e), kb = __shfl_sync(FULL, mine, 4 * c + 16 + 2 * t + e);
          pb[0][e] = __byte_perm(ka, kb, sel);
        }
      } else {
#pragma unroll
      for (int x = 0; x < X; ++x) {
        uint32_t hi, lo;
        split2(s[x][2 * t], s[x][2 * t + 1], &hi, &lo);
        const uint32_t ha = __shfl_sync(FULL, hi, from), hb = __shfl_sync(FULL, hi, from + 16);
        const uint32_t la = __shfl_sync(FULL, lo, from), lb = __shfl_sync(FULL, lo, from + 16);
        const uint32_t wa = (g & 1) ? la : ha, wb = (g & 1) ? lb : hb;
        pb[x][0] = __byte_perm(wa, wb, 0x5410);                      // keys c, c + 4
        pb[x][1] = __byte_perm(wa, wb, 0x7632);                      // keys c + 8, c + 12
      }
      }
      const auto v0 = load_piece<T::VB>(rows + 16 * t * T::RB), v1 = load_piece<T::VB>(rows + (16 * t + 4) * T::RB);
      const auto v2 = load_piece<T::VB>(rows + (16 * t + 8) * T::RB), v3 = load_piece<T::VB>(rows + (16 * t + 12) * T::RB);
      if constexpr (BITS == 4) {
#pragma unroll
        for (int h = 0; h < T::VD / 4; ++h) {                        // four columns of two keys share a word
          uint32_t p[4], q[4];
          nibbles(__byte_perm(v0.w[h >> 1], v1.w[h >> 1], (h & 1) ? 0x7632 : 0x5410), p);
          nibbles(__byte_perm(v2.w[h >> 1], v3.w[h >> 1], (h & 1) ? 0x7632 : 0x5410), q);
#pragma unroll
          for (int x = 0; x < X; ++x) {
            mma(o[2 * h][x], p[0], p[1], q[0], q[1], pb[x][0], pb[x][1]);
            mma(o[2 * h + 1][x], p[2], p[3], q[2], q[3], pb[x][0], pb[x][1]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < T::VD; i += 2) {
          uint32_t p[2], q[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t sel = (uint32_t)((i + e) & 3) | (uint32_t)(4 + ((i + e) & 3)) << 8;     // byte i + e of both, to bytes 0 and 2
            p[e] = centre(and_or(__byte_perm(v0.w[i >> 2], v1.w[i >> 2], sel), 0x00ff00ffu, 0x64006400u));
            q[e] = centre(and_or(__byte_perm(v2.w[i >> 2], v3.w[i >> 2], sel), 0x00ff00ffu, 0x64006400u));
          }
#pragma unroll
          for (int x = 0; x < X; ++x) mma(o[i / 2][x], p[0], p[1], q[0], q[1], pb[x][0], pb[x][1]);
        }
      }
    }
  }

  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int x = 0; x < X; ++x) {
#pragma unroll
      for (int w = ONE ? 1 : 4; w < 32; w <<= 1) l[x] += __shfl_xor_sync(FULL, l[x], w);
    }
  }
  // output column g VD + i of head 4 x + c, in units of sc
  __device__ __forceinline__ float value(int x, int i) const {
    return fmaf(o[i >> 1][x][2 * (i & 1) + 1], 1.f / kLo, o[i >> 1][x][2 * (i & 1)]);
  }
};

// BY_BLOCK false: a warp per `take` neighbouring units (all of a root, or one).  true: all warps of a cluster (of one block or more)
// work on one unit.
template <int BITS, int DP, int NH, bool BY_BLOCK>
__global__ void __launch_bounds__(32 * WARPS, DP * NH >= 256 ? 2 : DP >= 128 || DP * NH >= 128 ? 3 : 5) cached_attend_kernel(const AttendArgs a) {
  using T = Tile<BITS, DP>;
  constexpr int X = NH == 0 ? 1 : NH, GH = 4 * X;                                       // query heads of a unit
  constexpr int STAGE = 2 * T::TK * T::RB;                          // a tile's keys and values
  __shared__ double s_bounds[kMaxBuckets + 1];
  __shared__ __align__(128) uint8_t s_rows[WARPS][2 * STAGE];
  __shared__ __align__(16) uint32_t s_query[NH == 0 ? WARPS : 1][DP];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
  uint8_t* my = s_rows[wid];
  if (a.bias) {
    stage_bounds(s_bounds, a.bounds, a.buckets - 1, threadIdx.x, 32 * WARPS);
    __syncthreads();
  }
  int ranks = 1, rank = 0;
  if (BY_BLOCK) {
    ranks = (int)cg::this_cluster().num_blocks();
    rank = (int)cg::this_cluster().block_rank();
  }
  const uint32_t unit0 = BY_BLOCK ? blockIdx.x / (uint32_t)ranks : (blockIdx.x * WARPS + wid) * (uint32_t)a.take;
  if (unit0 >= a.units) return;                                     // (by warp: no barrier follows; by block: the grid fits)
  const int per_root = a.passes * a.kv_heads;
  const int64_t root = unit0 / (uint32_t)per_root;
  const int sub = (int)(unit0 - (uint32_t)root * (uint32_t)per_root);   // unit of the root: cached head, and which of its query heads
  Seen seen;
  int64_t first = a.first[root];
  int len = a.len[root];
  seen.t = a.bias ? a.times[root] : 0.0;
  if (first < 0 || len < 0 || len > 0x7fffffff - 64 || first > a.rows - len) {   // (a tile's last index stays within int32)
    if (lane == 0) atomicMax(a.status, 4);
    first = len = 0;
  }
  const int lo = len > a.window ? len - a.window : 0;
  seen.ns = min(a.sinks, lo);
  seen.n = len - lo + seen.ns;
  seen.skip = lo - seen.ns;
  const int tiles = (seen.n + T::TK - 1) / T::TK;
  const int worker = BY_BLOCK ? rank * WARPS + wid : 0, workers = BY_BLOCK ? ranks * WARPS : 1;
  Walk<BITS, DP, NH> w;
  int kv = sub / a.passes, pass = sub - kv * a.passes;
  constexpr int CPR = T::RB / 16;
  seen.k = a.k_codes + first * a.k_code_stride + 16 * (lane % CPR) + kv * T::RB;
  seen.v = a.v_codes + first * a.v_code_stride + 16 * (lane % CPR) + kv * T::RB;
  seen.ks = a.k_scales + first * a.k_scale_stride + 2 * kv;
  seen.vs = a.v_scales + first * a.v_scale_stride + 2 * kv;
  seen.ts = a.ts + first;
  const uint32_t to = (uint32_t)__cvta_generic_to_shared(my) + 16 * lane;
  for (int left = BY_BLOCK ? 1 : a.take; left > 0; --left) {
    const int head0 = kv * a.group + pass * GH, nh = NH == 0 ? 1 : min(GH, a.group - pass * GH);
    const float* bias = a.bias ? a.bias + (int64_t)head0 * a.buckets : &no_bias;
    if (worker < tiles) {
      // two tiles on their way: the query is prepared, and each tile worked on, while the next comes
      Rows<BITS, DP, NH == 0> next;
      next.load(a, seen, worker, to);
      asm volatile("cp.async.commit_group;" ::: "memory");
      if constexpr (NH == 0) w.begin_one(a, root, head0, s_query[wid]);
      else w.begin(a, root, head0, nh);
      int buf = 0, bucket = 0;                                      // (without a bias: bucket 0 of none)
      for (int tile = worker; tile < tiles; tile += workers) {
        const uint32_t scales = next.scales;
        if (a.bias) bucket = bucket_near(s_bounds, a.buckets - 1, seen.t - next.ts, bucket);
        if (tile + workers < tiles) next.load(a, seen, tile + workers, to + (buf ^ STAGE));
        asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 1;" ::: "memory");
        __syncwarp();
        w.tile(a, bias, seen, scales, bucket, my + buf, tile * T::TK, nh);
        __syncwarp();                                               // the tile's rows may be written over
        buf ^= STAGE;
      }
      w.finish();
    } else {
      w.none();
    }
    if constexpr (!BY_BLOCK) {
#pragma unroll
      for (int x = 0; x < X; ++x) {
        const int h = 4 * x + c;
        const float f = w.l[x] == 0.f ? 0.f : w.sc[x] * rcp_fast(w.l[x]);      // nothing seen, or nothing but -infinity: zeros
        const int64_t base = (root * a.heads + head0 + h) * a.dim;
        if (h < nh) {
#pragma unroll
          for (int i = 0; i < T::VD; i += 2) {
            const int e = g * T::VD + i;
            if (a.pairs) {
              if (e < a.dim) store_pair(a, base + e, w.value(x, i) * f, w.value(x, i + 1) * f);
            } else {
              if (e < a.dim) store_out(a, base + e, w.value(x, i) * f);
              if (e + 1 < a.dim) store_out(a, base + e + 1, w.value(x, i + 1) * f);
            }
          }
        }
      }
      if (++pass == a.passes) {                                      // the unit behind
        pass = 0;
        ++kv;
        seen.k += T::RB;
        seen.v += T::RB;
        seen.ks += 2;
        seen.vs += 2;
      }
    }
  }
  if constexpr (BY_BLOCK) {
    const int head0 = kv * a.group + pass * GH, nh = NH == 0 ? 1 : min(GH, a.group - pass * GH);
    __shared__ float s_m[WARPS][GH], s_l[WARPS][GH], b_m[GH], b_l[GH];
    static_assert(sizeof(s_rows) >= sizeof(float[WARPS][GH][DP + 4]), "the partial outputs take the rows' place");
    float(*s_o)[GH][DP + 4] = reinterpret_cast<float(*)[GH][DP + 4]>(&s_rows[0][0]);
    __syncthreads();                                                 // all warps are done with their rows
#pragma unroll
    for (int x = 0; x < X; ++x) {
#pragma unroll
      for (int i = 0; i < T::VD; ++i) s_o[wid][4 * x + c][g * T::VD + i] = w.value(x, i) * w.sc[x];
      if (g == 0) { s_m[wid][4 * x + c] = w.m[x]; s_l[wid][4 * x + c] = w.l[x]; }
    }
    __syncthreads();
    // the block's sums, at the block's maximum
    for (int i = threadIdx.x; i < nh * DP; i += 32 * WARPS) {
      const int h = i / DP, e = i - h * DP;
      float top = -INFINITY;
#pragma unroll
      for (int x = 0; x < WARPS; ++x) top = fmaxf(top, s_m[x][h]);
      const float base = top == -INFINITY ? 0.f : top;
      float o = 0.f, l = 0.f;
#pragma unroll
      for (int x = 0; x < WARPS; ++x) {
        const float f = exp2_fast((s_m[x][h] - base) * kLog2e);
        o = fmaf(s_o[x][h][e], f, o);
        l = fmaf(s_l[x][h], f, l);
      }
      if (ranks == 1) {
        if (e < a.dim) store_out(a, (root * a.heads + head0 + h) * a.dim + e, l == 0.f ? 0.f : o / l);
      } else {
        s_o[0][h][e] = o;                                            // this thread alone reads and writes column e of head h
        if (e == 0) { b_m[h] = top; b_l[h] = l; }
      }
    }
    if (ranks == 1) return;
    cg::cluster_group cl = cg::this_cluster();
    cl.sync();
    // every block finishes a part of the columns from all blocks' sums, in the order of their ranks
    for (int i = rank * (32 * WARPS) + threadIdx.x; i < nh * DP; i += ranks * (32 * WARPS)) {
      const int h = i / DP, e = i - h * DP;
      if (e >= a.dim) continue;
      float top = -INFINITY;
      for (int r = 0; r < ranks; ++r) top = fmaxf(top, *cl.map_shared_rank(&b_m[h], r));
      const float base = top == -INFINITY ? 0.f : top;
      float o = 0.f, l = 0.f;
      for (int r = 0; r < ranks; ++r) {
        const float f = exp2_fast((*cl.map_shared_rank(&b_m[h], r) - base) * kLog2e);
        o = fmaf(*cl.map_shared_rank(&s_o[0][h][e], r), f, o);
        l = fmaf(*cl.map_shared_rank(&b_l[h], r), f, l);
      }
      store_out(a, (root * a.heads + head0 + h) * a.dim + e, l == 0.f ? 0.f : o / l);
    }
    cl.sync();                                                       // no block leaves while its memory is read
  }
}

// Launches over `roots` roots whose windows have up to `tiles` tiles.
template <int BITS, int DP, int NH>
cudaError_t launch(AttendArgs& a, int64_t roots, int64_t tiles, cudaStream_t s) {
  const auto by_block = cached_attend_kernel<BITS, DP, NH, true>;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.blockDim = dim3(32 * WARPS);
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  auto of = [&](int ranks) {
    cfg.gridDim = dim3(a.units * (unsigned)ranks);
    at[0].val.clusterDim.x = (unsigned)ranks;
  };
  // Above the portable size a cluster has to be allowed, per kernel and device, and a device (or the part of it that the context has) may hold none.
  auto fits = [&](int ranks) {
    of(ranks);
    int clusters = 0;
    const bool ok = cudaFuncSetAttribute(by_block, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                    cudaOccupancyMaxActiveClusters(&clusters, by_block, &cfg) == cudaSuccess && clusters > 0;
    if (!ok) cudaGetLastError();
    return ok;
  };
  const AttendShape sh = choose_attend_shape(roots, a.kv_heads * a.passes, tiles, num_sms(), fits);
  a.take = sh.take;
  if (!sh.by_block) {
    const unsigned per = (unsigned)(WARPS * a.take);
    cached_attend_kernel<BITS, DP, NH, false><<<(a.units + per - 1) / per, 32 * WARPS, 0, s>>>(a);
    return cudaGetLastError();
  }
  of(sh.ranks);
  return cudaLaunchKernelEx(&cfg, by_block, (const AttendArgs)a);
}

template <int BITS, int DP>
cudaError_t launch_heads(AttendArgs& a, int64_t roots, int64_t tiles, cudaStream_t s) {
  return a.group > 4 ? launch<BITS, DP, 2>(a, roots, tiles, s) : a.group > 1 ? launch<BITS, DP, 1>(a, roots, tiles, s) : launch<BITS, DP, 0>(a, roots, tiles, s);
}

template <int BITS>
cudaError_t launch_dim(AttendArgs& a, int64_t roots, int64_t tiles, cudaStream_t s) {
  switch (padded_dim(a.dim)) {
    case 32: return launch_heads<BITS, 32>(a, roots, tiles, s);
    case 64: return launch_heads<BITS, 64>(a, roots, tiles, s);
    default: return launch_heads<BITS, 128>(a, roots, tiles, s);
  }
}

}  // namespace

extern "C" int tgnn_cached_attend(const void* q, int dtype, const tgnn_cache* k_host, const tgnn_cache* v_host, int64_t n, int heads,
                                  const int64_t* first, const int32_t* len, const float* bias, int num_buckets, const double* bounds,
                                  const double* times, const double* ts, int window, int sinks, int max_len, float scale, void* out,
                                  int32_t* status, void* stream, char* err_host, int64_t err_size) {
  const char* who = "tgnn_cached_attend";
  CacheView k, v;
  int rc = check_cache(who, "k", k_host, &k, err_host, err_size);
  if (!rc) rc = check_cache(who, "v", v_host, &v, err_host, err_size);
  if (rc) return rc;
  if (k.rows != v.rows || k.heads != v.heads || k.dim != v.dim || k.bits != v.bits)
    return fail(err_host, err_size, TGNN_ESHAPE, "%s: k and v differ in rows, heads, dim or bits", who);
  if (!known_dtype(dtype)) return fail(err_host, err_size, TGNN_EINVAL, "%s: unknown type %d", who, dtype);
  if (n < 0 || window < 0 || sinks < 0 || (int64_t)window + sinks < 1 || max_len < 0)
    return fail(err_host, err_size, TGNN_EINVAL, "%s: size out of range (window and sinks see one entry at least)", who);
  if (heads < 1 || heads > 1024 || heads % k.heads)
    return fail(err_host, err_size, TGNN_EINVAL, "%s: %d heads over %d cached ones", who, heads, k.heads);
  if (!status || (n > 0 && (!q || !out || !first || !len))) return fail(err_host, err_size, TGNN_EINVAL, "%s: null pointer", who);
  if (bias && (num_buckets < 1 || num_buckets > kMaxBuckets))
    return fail(err_host, err_size, TGNN_EINVAL, "%s: %d buckets (1 to %d)", who, num_buckets, kMaxBuckets);
  if (bias && n > 0 && ((num_buckets > 1 && !bounds) || !times || (k.rows > 0 && !ts)))
    return fail(err_host, err_size, TGNN_EINVAL, "%s: a bias needs bounds, times and ts", who);
  const int es = elem_bytes(dtype) - 1;
  if ((((uintptr_t)q | (uintptr_t)out) & es) || (((uintptr_t)first | (uintptr_t)bounds | (uintptr_t)times | (uintptr_t)ts) & 7) ||
      (((uintptr_t)len | (uintptr_t)bias | (uintptr_t)status) & 3))
    return fail(err_host, err_size, TGNN_EINVAL, "%s: a pointer is not aligned to its element", who);
  AttendArgs a = {};
  a.group = heads / k.heads;
  a.passes = a.group > 4 ? (a.group + 7) / 8 : 1;
  if (n > 0x0fffffff / ((int64_t)k.heads * a.passes)) return fail(err_host, err_size, TGNN_ECAPACITY, "%s: n * heads above 2^28", who);
  if (n == 0) return TGNN_OK;
  a.q = q;
  a.out = out;
  a.dtype = dtype;
  a.k_codes = k.codes;
  a.v_codes = v.codes;
  a.k_scales = k.scales;
  a.v_scales = v.scales;
  a.k_code_stride = (uint32_t)k.code_stride;
  a.v_code_stride = (uint32_t)v.code_stride;
  a.k_scale_stride = (uint32_t)k.scale_stride;
  a.v_scale_stride = (uint32_t)v.scale_stride;
  a.rows = k.rows;
  a.heads = heads;
  a.kv_heads = k.heads;
  a.dim = k.dim;
  a.units = (uint32_t)(n * k.heads * a.passes);
  a.first = first;
  a.len = len;
  a.bias = bias;
  a.bounds = bounds;
  a.times = times;
  a.ts = ts;
  a.buckets = bias ? num_buckets : 0;
  a.window = window;
  a.sinks = sinks;
  a.scale = scale;
  a.status = status;
  int64_t see = (int64_t)window + sinks;
  if (max_len > 0 && max_len < see) see = max_len;
  if (k.rows < see) see = k.rows;
  const int tk = k.bits * padded_dim(k.dim) >= 1024 ? 16 : 32;
  const int64_t tiles = (see + tk - 1) / tk;
  a.pairs = k.dim % 2 == 0 && (((uintptr_t)q | (uintptr_t)out) & (2 * es + 1)) == 0;
  const cudaError_t e = k.bits == 4 ? launch_dim<4>(a, n, tiles, (cudaStream_t)stream) : launch_dim<8>(a, n, tiles, (cudaStream_t)stream);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return fail(err_host, err_size, TGNN_ECUDA, "%s: %s", who, cudaGetErrorString(e));
  }
  return TGNN_OK;
}
